// Batched field product Y_hat[b] = M x_hat[b] over F_q on the tcgen05 tensor
// cores (the server's online work at batch > 1, Sec. 6.1).
//
// Arithmetic.  Each centred x_hat entry is split into four signed base-256
// digits d_k in [-128, 127] (x = sum_k 2^(8k) d_k), so
//     (M x_hat)_i = sum_k 2^(8k) sum_j M_ij d_k[j]        (exact over Z).
// The inner sums run on the tensor cores as an fp16 GEMM (every int8 weight
// and every digit is an exact fp16 value) with fp32 accumulation in TMEM.  A
// product is at most 128 * 128 = 2^14 in magnitude, so a chunk of 1024
// K-elements sums to at most 2^24: every partial sum is an integer that fp32
// holds exactly.  After each chunk the epilogue warps read the accumulator,
// convert it to integers, combine the four digits in int64, reduce mod q and
// add to a running sum per output.  (This GPU generation has no int8 tcgen05
// kind; fp16 and bf16 run at the same rate, and int8 -> fp16 is one byte
// permute and one packed add per two elements.)
//
// Tiles.  Two CTAs on two SMs (a CTA pair of a cluster) run one MMA of
// M = 256 rows of M by N = 256 digit rows (64 vectors x 4 digits, the digit
// rows of vector v at N-rows 4v..4v+3) with tcgen05 cta_group::2: each CTA
// holds its own 128 rows of M and half of the digit rows (vectors 0-31 in the
// even CTA, 32-63 in the odd one), and each CTA's TMEM receives the full
// 128 x 256 accumulator of its own rows.  The even CTA issues the MMAs.
// K may further be split over pairs of the cluster; their mod-q partial sums
// are added through distributed shared memory, each rank finishing a slice
// of the vectors.
//
// Warp roles (608 threads per CTA, 19 warps):
//   warps 0-7    convert the int8 M tile to fp16 in the 128-byte-swizzled
//                K-major layout the MMA reads: warps 0-3 take the even
//                K-blocks, warps 4-7 the odd ones (four threads per row);
//   warps 8-11   epilogue for vectors 0-31, warps 12-15 for vectors 32-63
//                (TMEM lanes 32 (w mod 4) .. +31);
//   warp 16      bulk-copies this CTA's half of the digit operand;
//   warp 17      allocates TMEM; in the even CTA it issues the MMAs, in
//                the odd CTA one lane tells the even CTA when a stage of
//                its own shared memory is filled;
//   warp 18      streams 128 x 64 int8 tiles of M into a ring of raw tiles
//                with the tensor memory accelerator (TMA), far ahead of the
//                converter.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cstring>
#include <map>
#include <mutex>
#include <tuple>
#include <vector>

#include "common.cuh"
#include "launch.h"
#include "tensor.cuh"

namespace cg = cooperative_groups;

namespace pv {
namespace {

constexpr int kBM = 128;            // rows of M per CTA
constexpr int kBV = 64;             // vectors per CTA
constexpr int kBN = 4 * kBV;        // MMA N (digit rows)
constexpr int kBK = 64;             // K-elements per stage (128 bytes of fp16)
constexpr int kStages = 5;
constexpr int kRaw = 8;                 // raw int8 tiles of M in flight
constexpr int kChunkBlocks = 16;    // 16 x 64 = 1024 K-elements per exact chunk
constexpr int kATile = kBM * kBK * 2;   // 16 KiB
constexpr int kBTile = kBN * kBK * 2;   // 32 KiB
constexpr int kBHalf = kBTile / 2;     // 16 KiB: the digit rows one CTA of a pair holds
constexpr int kStageBytes = kATile + kBHalf;
constexpr int kThreads = 608;
constexpr int kConvThreads = 256;   // warps 0-7
constexpr int kEpiThreads = 256;    // warps 8-15
constexpr int kWarpLoader = 16, kWarpMma = 17, kWarpWLoad = 18;
constexpr int kRawTile = kBM * kBK;     // 8 KiB: rows of 64 bytes, unswizzled
constexpr int kRawOff = kStages * kStageBytes;
constexpr int kMmaSmem = kRawOff + kRaw * kRawTile + 1024;  // + alignment slack

// Arrival on a barrier of any CTA of the cluster (address from mapa).
__device__ __forceinline__ uint32_t cluster_addr(const void *p, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}

// ---------------------------------------------------------------- async copies, fences
__device__ __forceinline__ void bulk_g2s(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
            smem_addr(dst)),
        "l"(src), "r"(bytes), "r"(smem_addr(bar))
        : "memory");
}
// 2-D tiled TMA load of box {x .. x+63, y .. y+127} into shared memory;
// elements outside the tensor arrive as zeros.
__device__ __forceinline__ void tma_load_2d(void *dst, const CUtensorMap *map, int x, int y, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            smem_addr(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_addr(bar))
        : "memory");
}
// ---------------------------------------------------------------- tcgen05
// Instruction descriptor, kind::f16: fp16 A and B (format 0), f32 D (1),
// both K-major, N = 256, M = 256 (the pair's two 128-row halves).
constexpr uint32_t kIdesc = (1u << 4) | (0u << 7) | (0u << 10) | ((uint32_t)(kBN >> 3) << 17) |
                            ((uint32_t)(2 * kBM >> 4) << 24);

__device__ __forceinline__ void mma_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc,
                                         uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(tmem_d),
        "l"(adesc), "l"(bdesc), "r"(kIdesc), "r"(accumulate));
}
// Arrive on `bar` (same offset) in every CTA of `mask` once all MMAs issued
// so far (by this lane) have completed.
__device__ __forceinline__ void mma_commit_pair(uint64_t *bar, uint16_t mask) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            smem_addr(bar)),
        "h"(mask)
        : "memory");
}
__device__ __forceinline__ void warp_commit_pair(uint64_t *bar, uint16_t mask) {
    if (elect_one()) mma_commit_pair(bar, mask);
    __syncwarp();
}
// Four signed bytes -> two fp16x2 words holding the same integers: with
// u = b + 128 (the byte xor 0x80), the fp16 pattern 0x6400 | u is 1024 + u,
// and subtracting 1152 leaves b exactly.
__device__ __forceinline__ void i8x4_to_f16x4(uint32_t w, uint32_t &lo, uint32_t &hi) {
    const uint32_t u = w ^ 0x80808080u;
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x5150);  // bytes u0, 0x64, u1, 0x64
    const uint32_t b = __byte_perm(u, 0x64646464u, 0x5352);  // bytes u2, 0x64, u3, 0x64
    const __half2 off = __halves2half2(__ushort_as_half(0xE480u), __ushort_as_half(0xE480u));  // -1152
    const __half2 ha = __hadd2(*reinterpret_cast<const __half2 *>(&a), off);
    const __half2 hb = __hadd2(*reinterpret_cast<const __half2 *>(&b), off);
    lo = *reinterpret_cast<const uint32_t *>(&ha);
    hi = *reinterpret_cast<const uint32_t *>(&hb);
}
__device__ __forceinline__ uint32_t f16x2_of_int(int lo, int hi) {
    const __half2 v = __halves2half2(__int2half_rn(lo), __int2half_rn(hi));
    return *reinterpret_cast<const uint32_t *>(&v);
}

// ---------------------------------------------------------------- epilogue arithmetic
// Four exact digit-plane sums s_l (|s_l| <= 2^24, one chunk) -> 
//     (s_0 + 2^8 s_1 + 2^16 s_2 + 2^24 s_3) * 2^-32 mod q,
// in [0, q).  The combination is formed in int64 (|.| < 2^48.01) and shifted
// by K0 = 2^18 q (> 2^48.01, a multiple of q) to u in (0, 2^50); Montgomery's
// REDC with R = 2^32 then gives (u + m q) / 2^32 < 2^18 + q < 2q, where
// m = -u q^-1 mod 2^32, and one conditional subtraction finishes.  The factor
// 2^-32 is the same for every term of an output's sum and is removed once,
// after the last chunk (kR2 below).
constexpr int64_t kK0 = (int64_t)PVMVMD_Q << 18;
__device__ __forceinline__ uint32_t digits_redc(int s0, int s1, int s2, int s3) {
    const uint64_t u = (uint64_t)((int64_t)s0 + kK0 + (int64_t)s1 * 256 + (int64_t)s2 * 65536 +
                                  (int64_t)s3 * 16777216);
    const uint32_t m = (uint32_t)u * kQInvNeg;
    const uint32_t r = (uint32_t)((u + (uint64_t)m * kQ) >> 32);
    return r >= kQ ? r - kQ : r;
}
// R^2 mod q for R = 2^32: fmul_mont(x, kR2) = x R mod q undoes the 2^-32.
constexpr uint32_t kRmodQ = (uint32_t)((1ull << 32) % PVMVMD_Q);
constexpr uint32_t kR2 = (uint32_t)(((uint64_t)kRmodQ * kRmodQ) % PVMVMD_Q);

// ---------------------------------------------------------------- digit operand
// X_hat (B x K u32) -> pre-tiled fp16 digit operand: for vector tile nt and
// K-block kb, a 32 KiB block laid out exactly as the MMA's B tile in shared
// memory.  Zero for vectors >= B and K-elements >= K.  One thread per
// (vector, 8 K-elements).
__global__ void __launch_bounds__(256) k_digit_tiles(const uint32_t *__restrict__ Xhat, int B, int K,
                                                    int nkb, int nvt, uint8_t *__restrict__ D) {
    // the product kernel may start its set-up now; it reads these tiles only
    // after griddepcontrol.wait
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const size_t gid = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    const size_t per_vec = (size_t)nkb * 8;  // 8-element groups per vector
    const size_t total = (size_t)nvt * kBV * per_vec;
    if (gid >= total) return;
    const int v = (int)(gid / per_vec);
    const int grp = (int)(gid % per_vec);
    const int kb = grp >> 3, chunk = grp & 7;
    const int k0 = kb * kBK + chunk * 8;
    int d[4][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int k = k0 + e;
        if (v < B && k < K) {
            limb_split(Xhat[(size_t)v * K + k], d[0][e], d[1][e], d[2][e], d[3][e]);
        } else {
            d[0][e] = d[1][e] = d[2][e] = d[3][e] = 0;
        }
    }
    const int nt = v / kBV, vl = v % kBV;
    uint8_t *blk = D + ((size_t)nt * nkb + kb) * kBTile;
#pragma unroll
    for (int l = 0; l < 4; ++l) {
        const uint32_t row = 4 * vl + l;
        uint4 q;
        q.x = f16x2_of_int(d[l][0], d[l][1]);
        q.y = f16x2_of_int(d[l][2], d[l][3]);
        q.z = f16x2_of_int(d[l][4], d[l][5]);
        q.w = f16x2_of_int(d[l][6], d[l][7]);
        *reinterpret_cast<uint4 *>(blk + sw128_off(row, chunk)) = q;
    }
}

// ---------------------------------------------------------------- main kernel
template <bool kVec>
__global__ void __launch_bounds__(kThreads, 1)
    k_batched(const __grid_constant__ CUtensorMap tmap_w, const int8_t *__restrict__ W, int m, int K,
              const uint8_t *__restrict__ D, int nkb, int B, uint32_t *__restrict__ Yhat,
              uint32_t *__restrict__ err, int skip_report, uint64_t wait_ns) {
    cg::cluster_group cluster = cg::this_cluster();
    extern __shared__ uint8_t smem_raw[];
    // full: this CTA's stage is complete -- the converter group's warps have
    // arrived, the digit half has landed (transaction bytes) and, in the even
    // CTA, the odd CTA has reported its own stage complete;
    // empty: the pair's MMAs on the stage finished (commit from the even CTA);
    // acc_full / acc_empty: the accumulator buffer is ready / drained by the
    // epilogue warps of both CTAs (arrivals land in the even CTA).
    __shared__ __align__(8) uint64_t full[kStages], empty_bar[kStages];
    __shared__ __align__(8) uint64_t acc_full[2], acc_empty[2], mma_done;
    __shared__ __align__(8) uint64_t raw_full[kRaw], raw_empty[kRaw];  // raw int8 tile ring
    __shared__ uint32_t s_tmem;

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(kFull, tid >> 5, 0);  // uniform, so that the roles' operands are
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - smem_addr(smem_raw));

    const int m0 = blockIdx.x * kBM;
    const int nt = blockIdx.y;
    const uint32_t rank = cluster.block_rank();  // = (blockIdx.x & 1) + 2 * blockIdx.z
    const uint32_t half = rank & 1u;             // 0: the even CTA, which issues the MMAs
    const uint32_t leader = rank & ~1u;
    const uint16_t pair_mask = (uint16_t)(3u << leader);
    const int split = (int)cluster.num_blocks() / 2;
    const int zr = (int)(rank >> 1);
    const int per = (nkb + split - 1) / split;
    const int kb0 = zr * per;
    const int kb1 = min(nkb, kb0 + per);
    const int nblk = max(0, kb1 - kb0);
    const int nchunks = (nblk + kChunkBlocks - 1) / kChunkBlocks;

    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) {
            // the warps of one converter group + the digit copy's arrival
            // (+ the odd CTA's report, in the even CTA)
            mbar_init(&full[s], kConvThreads / 64 + 1 + (half == 0 ? 1 : 0));
            mbar_init(&empty_bar[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&acc_full[b], 1);
            mbar_init(&acc_empty[b], 2 * kEpiThreads / 32);  // epilogue warps of both CTAs
        }
        mbar_init(&mma_done, 1);
        for (int r = 0; r < kRaw; ++r) {
            mbar_init(&raw_full[r], 1);
            mbar_init(&raw_empty[r], kConvThreads / 64);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kWarpMma) {  // one warp of each CTA of the pair allocates together
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(
                         smem_addr(&s_tmem)));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    tc_fence_before();
    cluster.sync();  // barriers initialised and TMEM allocated in every CTA
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    uint32_t run[32];  // epilogue: running sums of 32 vectors for one row, times 2^-32 mod q
#pragma unroll
    for (int v = 0; v < 32; ++v) run[v] = 0u;

    if (warp < 8) {
        // ------------------------------------------------ A: int8 M tile -> fp16 swizzled
        // Two groups of four warps take alternate K-blocks.  In a block,
        // thread t of a group converts 16 K-elements (two 16-byte fp16
        // chunks) of rows t/4 + 32 j, j = 0..3: a quarter-warp covers one
        // row's 64 bytes.
        const int grp = warp >> 2;
        const int t = tid & 127;
        const int r0 = t >> 2, qk = t & 3;
        auto convert_store = [&](uint8_t *a, const uint4 (&v)[4]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {  // 16 int8 -> two 16-byte fp16 chunks
                uint32_t o[8];
                i8x4_to_f16x4(v[j].x, o[0], o[1]);
                i8x4_to_f16x4(v[j].y, o[2], o[3]);
                i8x4_to_f16x4(v[j].z, o[4], o[5]);
                i8x4_to_f16x4(v[j].w, o[6], o[7]);
                const int row = r0 + 32 * j;
                *reinterpret_cast<uint4 *>(a + sw128_off(row, 2 * qk)) = make_uint4(o[0], o[1], o[2], o[3]);
                *reinterpret_cast<uint4 *>(a + sw128_off(row, 2 * qk + 1)) = make_uint4(o[4], o[5], o[6], o[7]);
            }
        };
        if constexpr (kVec) {
            // the int8 tile arrives by TMA (warp 18)
            for (int i = grp; i < nblk; i += 2) {
                const int s = i % kStages, rs = i % kRaw;
                const uint32_t ph = (uint32_t)(i / kStages) & 1u, rph = (uint32_t)(i / kRaw) & 1u;
                if (!mbar_wait_warp(&raw_full[rs], rph, err, wait_ns) || !mbar_wait_warp(&empty_bar[s], ph ^ 1u, err, wait_ns))
                    break;
                const uint8_t *raw = smem + kRawOff + rs * kRawTile;
                uint4 v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    v[j] = *reinterpret_cast<const uint4 *>(raw + (r0 + 32 * j) * kBK + 16 * qk);
                convert_store(smem + s * kStageBytes, v);
                fence_async_smem();  // this thread's stores -> visible to the tensor cores
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&full[s]);
                    mbar_arrive(&raw_empty[rs]);
                }
            }
        } else {
            // rows of any length and alignment, from the words that hold them,
            // a block ahead (bytes past K meet zero digits)
            const int8_t *W_end = W + (size_t)m * K;
            auto fetch = [&](int i, uint4 (&v)[4]) {
                const int k0 = (kb0 + i) * kBK + 16 * qk;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int grow = m0 + r0 + 32 * j;
                    v[j] = i < nblk && grow < m && k0 < K ? load16_any(W + (size_t)grow * K + k0, W, W_end)
                                                          : make_uint4(0u, 0u, 0u, 0u);
                }
            };
            uint4 next[4];
            fetch(grp, next);
            for (int i = grp; i < nblk; i += 2) {
                const int s = i % kStages;
                const uint32_t ph = (uint32_t)(i / kStages) & 1u;
                uint4 v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = next[j];
                fetch(i + 2, next);
                if (!mbar_wait_warp(&empty_bar[s], ph ^ 1u, err, wait_ns)) break;
                convert_store(smem + s * kStageBytes, v);
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&full[s]);
            }
        }
    } else if (warp < 16) {
        // ------------------------------------------------ epilogue: TMEM -> mod-q sums
        const int q = warp & 3;            // TMEM lane quadrant
        const int grp = (warp - 8) >> 2;   // vectors 32 grp .. 32 grp + 31
        const uint32_t acc_empty_leader = cluster_addr(&acc_empty[0], leader);
        for (int c = 0; c < nchunks; ++c) {
            const int bsel = c & 1;
            if (!mbar_wait_warp(&acc_full[bsel], (uint32_t)(c >> 1) & 1u, err, wait_ns)) break;
            tc_fence_after();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t r[32];
                tmem_ld32(tmem + ((uint32_t)(32 * q) << 16) + (uint32_t)(bsel * kBN + 128 * grp + 32 * j), r);
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    run[8 * j + v] = fadd(run[8 * j + v],
                                          digits_redc(__float2int_rn(__uint_as_float(r[4 * v])),
                                                      __float2int_rn(__uint_as_float(r[4 * v + 1])),
                                                      __float2int_rn(__uint_as_float(r[4 * v + 2])),
                                                      __float2int_rn(__uint_as_float(r[4 * v + 3]))));
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(acc_empty_leader + 8u * (uint32_t)bsel);
        }
    } else if (warp == kWarpLoader) {
        // ------------------------------------------------ B: this CTA's digit half
        if (lane == 0) {
            const uint8_t *src = D + ((size_t)nt * nkb + kb0) * kBTile + (size_t)half * kBHalf;
            // the digit tiles come from the kernel launched just before this one
            asm volatile("griddepcontrol.wait;" ::: "memory");
            int issued = 0;
            for (int i = 0; i < nblk; ++i) {
                const int s = i % kStages;
                const uint32_t ph = (uint32_t)(i / kStages) & 1u;
                if (!mbar_wait(&empty_bar[s], ph ^ 1u, err, wait_ns)) break;
                uint8_t *b = smem + s * kStageBytes + kATile;
                mbar_arrive_tx(&full[s], kBHalf);
                bulk_g2s(b, src + (size_t)i * kBTile, kBHalf, &full[s]);
                issued = i + 1;
            }
            // copies in flight complete before the CTA may exit
            for (int i = max(0, issued - kStages); i < issued; ++i)
                mbar_wait(&full[i % kStages], (uint32_t)(i / kStages) & 1u, err, wait_ns);
        }
    } else if (warp == kWarpWLoad) {
        // ------------------------------------------------ raw int8 tiles of M by TMA
        if (kVec && lane == 0) {
            int issued = 0;
            for (int i = 0; i < nblk; ++i) {
                const int rs = i % kRaw;
                const uint32_t rph = (uint32_t)(i / kRaw) & 1u;
                if (!mbar_wait(&raw_empty[rs], rph ^ 1u, err, wait_ns)) break;
                mbar_arrive_tx(&raw_full[rs], kRawTile);
                tma_load_2d(smem + kRawOff + rs * kRawTile, &tmap_w, (kb0 + i) * kBK, m0, &raw_full[rs]);
                issued = i + 1;
            }
            // copies in flight complete before the CTA may exit
            for (int i = max(0, issued - kRaw); i < issued; ++i)
                mbar_wait(&raw_full[i % kRaw], (uint32_t)(i / kRaw) & 1u, err, wait_ns);
        }
    } else if (half == 0) {
        // ------------------------------------------------ MMA issuer (even CTA)
        {
            bool ok = true;
            for (int c = 0; c < nchunks && ok; ++c) {
                const int bsel = c & 1;
                if (!mbar_wait_warp(&acc_empty[bsel], ((uint32_t)(c >> 1) & 1u) ^ 1u, err, wait_ns)) break;
                tc_fence_after();
                const uint32_t dcol = tmem + (uint32_t)(bsel * kBN);
                const int i_end = min(nblk, (c + 1) * kChunkBlocks);
                for (int i = c * kChunkBlocks; i < i_end; ++i) {
                    const int s = i % kStages;
                    const uint32_t ph = (uint32_t)(i / kStages) & 1u;
                    if (!mbar_wait_warp(&full[s], ph, err, wait_ns)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t ad = sw128_desc(base) + (uint32_t)(s * kStageBytes >> 4);
                    const uint64_t bd = ad + (uint32_t)(kATile >> 4);
                    if (elect_one()) {
                        mma_pair(dcol, ad, bd, i > c * kChunkBlocks ? 1u : 0u);
#pragma unroll
                        for (int k = 1; k < kBK / 16; ++k) mma_pair(dcol, ad + 2u * k, bd + 2u * k, 1u);
                        mma_commit_pair(&empty_bar[s], pair_mask);
                    }
                    __syncwarp();
                }
                warp_commit_pair(&acc_full[bsel], pair_mask);
            }
            // all issued MMAs have finished before TMEM is released
            warp_commit_pair(&mma_done, (uint16_t)(1u << leader));
            mbar_wait_warp(&mma_done, 0, err, wait_ns);
        }
    } else {
        // ------------------------------------------------ stage relay (odd CTA)
        if (lane == 0) {
            const uint32_t full_leader = cluster_addr(&full[0], leader);
            for (int i = 0; i < nblk; ++i) {
                const int s = i % kStages;
                const uint32_t ph = (uint32_t)(i / kStages) & 1u;
                if (!mbar_wait(&full[s], ph, err, wait_ns)) break;
                // a failure-path test withholds one report, so that the even
                // CTA's wait for this stage expires (off: skip_report < 0)
                if (i == skip_report) continue;
                mbar_arrive_cluster(full_leader + 8u * (uint32_t)s);
            }
        }
    }

    // ---------------------------------------------------- split-K reduction and store
    tc_fence_before();
    __syncthreads();  // this CTA's roles are done
    cluster.sync();   // ... and the peer's: no MMA reads this CTA's stages any more
    uint32_t *part = reinterpret_cast<uint32_t *>(smem);  // [kBV][kBM] mod-q partial sums
    if (warp >= 8 && warp < 16) {
        const int row = 32 * (warp & 3) + lane;
        const int v0 = 32 * ((warp - 8) >> 2);
#pragma unroll
        for (int v = 0; v < 32; ++v) part[(v0 + v) * kBM + row] = run[v];
    }
    cluster.sync();
    // the CTA at K-rank zr finishes vectors [zr * 64 / split, (zr + 1) * 64 / split)
    const int vper = kBV / split;
    for (int idx = tid; idx < vper * kBM; idx += kThreads) {
        const int v = zr * vper + idx / kBM, row = idx % kBM;
        uint32_t sum = 0;
        for (int rr = 0; rr < split; ++rr)
            sum = fadd(sum, cluster.map_shared_rank(part, (unsigned)(2 * rr) + half)[v * kBM + row]);
        sum = fmul_mont(sum, kR2);
        const int b = nt * kBV + v, grow = m0 + row;
        if (grow < m && b < B) Yhat[(size_t)b * m + grow] = sum;
    }
    cluster.sync();
    if (warp == kWarpMma) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

// Resident clusters of (2, 1, split) CTAs of the kernel, from the occupancy
// calculator (a cluster must fit in one GPC), cached per (kernel, split,
// device).
int resident_clusters(const void *kern, int split) {
    static std::map<std::tuple<const void *, int, int>, int> cache;
    static std::mutex mu;
    int cur = 0;
    cudaGetDevice(&cur);
    std::lock_guard<std::mutex> lock(mu);
    int &c = cache[std::make_tuple(kern, split, cur)];
    if (c == 0) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(2, 1, split);
        cfg.blockDim = dim3(kThreads, 1, 1);
        cfg.dynamicSmemBytes = kMmaSmem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = split;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n <= 0) {
            (void)cudaGetLastError();
            int dev = 0, sms = 0;
            cudaGetDevice(&dev);
            cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
            n = max(1, sms / (2 * split));
        }
        c = n;
    }
    return c;
}

// Cluster split of K: the fewest pairs per tile that still give the fewest
// waves per unit of work, with at least 4 K-blocks per pair.
int choose_split(const void *kern, int pairs, int nkb) {
    int best = 1;
    double best_cost = 1e30;
    for (int split = 1; split <= 4; split *= 2) {
        if (split > 1 && nkb < 4 * split) break;
        const int clusters = pairs;  // one cluster of `split` pairs per tile pair
        const int cap = resident_clusters(kern, split);
        const int waves = (clusters + cap - 1) / cap;
        const double cost = (double)waves / split + 0.02 * (split - 1);
        if (cost < best_cost - 1e-9) {
            best_cost = cost;
            best = split;
        }
    }
    return best;
}

cudaError_t batched_launch(const int8_t *W, int m, int K, const uint32_t *Xhat, int B, uint32_t *Yhat,
                           uint32_t *err, uint8_t *D, cudaStream_t s) {
    const int nkb = (K + kBK - 1) / kBK;
    const int nvt = (B + kBV - 1) / kBV;
    const size_t threads = (size_t)nvt * kBV * nkb * 8;
    k_digit_tiles<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(Xhat, B, K, nkb, nvt, D); note_launch();
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const int mp = (m + 2 * kBM - 1) / (2 * kBM);  // CTA pairs along M
    // M as a K x m tensor of bytes for TMA: needs 16-byte aligned rows
    const bool vec = (K % 16 == 0) && ((reinterpret_cast<uintptr_t>(W) & 15u) == 0);
    CUtensorMap tmap;
    memset(&tmap, 0, sizeof(tmap));
    if (vec) {
        PFN_cuTensorMapEncodeTiled_v12000 encode = tensor_map_encoder();
        if (!encode) return cudaErrorNotSupported;
        const cuuint64_t gdim[2] = {(cuuint64_t)K, (cuuint64_t)m};
        const cuuint64_t gstride[1] = {(cuuint64_t)K};
        const cuuint32_t box[2] = {(cuuint32_t)kBK, (cuuint32_t)kBM};
        const cuuint32_t estride[2] = {1, 1};
        if (encode(&tmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t *>(W), gdim, gstride, box, estride,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    }
    auto kern = vec ? k_batched<true> : k_batched<false>;
    const cudaError_t a1 =
        func_attr((const void *)k_batched<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMmaSmem);
    const cudaError_t a2 =
        func_attr((const void *)k_batched<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMmaSmem);
    if (a1 != cudaSuccess) return a1;
    if (a2 != cudaSuccess) return a2;
    const int split = choose_split((const void *)kern, mp * nvt, nkb);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * mp, nvt, split);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = kMmaSmem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = split;
    // programmatic dependent launch: barrier set-up, TMEM allocation and the
    // first weight tiles overlap the digit-tile kernel
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const DebugWait dbg = debug_wait();
    const int skip_report = dbg.site == PVMVMD_DEBUG_WAIT_PRODUCT ? (int)dbg.index : -1;
    const uint64_t wait_ns = dbg.site == PVMVMD_DEBUG_WAIT_PRODUCT ? dbg.limit : kWaitNs;
    return counted_launch(cudaLaunchKernelEx(&cfg, kern, tmap, W, m, K, (const uint8_t *)D, nkb, B, Yhat, err, skip_report,
                              wait_ns));
}

// ---------------------------------------------------------------------------
// Grouped persistent product: one launch over a list of independent batched
// products (for example the projections of a decoder layer).  Work items are
// (job, pair of 128-row tiles, 64-vector tile, K-split); one CTA pair of a
// thread-block cluster stays resident and walks its items, its pipelines
// (stages, raw ring, TMEM accumulators) running on from one item to the next, so that the pipeline fill, TMEM allocation and barrier
// set-up are paid once per launch and an item's epilogue overlaps the next
// item's MMAs.  Items are ordered longest first (jobs by blocks per item),
// and within a job by row pair, then K-split, then vector tile, so that the
// items that run at the same time read the same rows of M; pair c of C takes
// items c, 2C - 1 - c, 2C + c, ... (a snake order, close to the greedy
// longest-first assignment).  A job whose K is split over several items
// adds its partial sums (each canonical, times R^2 already applied) into a
// 64-bit buffer with atomics; a final kernel reduces them mod q.  (Having
// the epilogue warp that adds the last part reduce its block instead, behind
// a fence and a counter, held the epilogue up and was slower: 8B layer
// 84 -> 97 us.)
//
// The converted M goes to TMEM, not to shared memory: a converter thread
// takes one row's 64 bytes of a K-block, writes the fp16 values to its TMEM
// lane, and the MMAs read A from there.  In shared memory M's K-block cost 128
// write and 128 read wavefronts of the about 710 that a 64-vector K-block came
// to, against 512 cycles of MMA, and left room for 3 stages and 4 raw tiles.
// TMEM holds M only if the accumulators leave columns: a 64-vector tile is
// computed as two parts of N = 128, whose exact chunks of 16 K-blocks end in
// turn every 8, so that three accumulators of 128 columns do where two of 256
// did, and the epilogue still reads one while the MMAs go on.  A ring of raw
// tiles that deep (96 or 160 KiB) needs no L2 prefetch beside it; the requests
// of that, from one lane, had held the loads up.
// One 8B-class layer for 64 vectors 84.7 -> 79.5 us, for 16 vectors 59.4 ->
// 46.4; one 70B-class layer for 256 vectors 1092 -> 1020 us (1.72 PFLOP/s of
// the four digits, at the power cap; a plain bf16 GEMM sustains 1.69).  Tiles of
// two K-blocks (128-byte rows) in the raw ring measured the same.
// ---------------------------------------------------------------------------
constexpr int kMaxGroupJobs = 8;
constexpr int kMaxSplit = 8;
constexpr int kNarrowMaxB = 16;  // batches up to this size use 16-vector tiles

// Tile geometry of the grouped kernel for V vectors per tile: 64 (256 digit
// rows, the batched configurations) or 16 (64, small batches, where a
// 64-vector tile would leave three quarters of the MMA idle).  A stage holds
// one K-block for each group of four converter warps: two for V = 64; four for
// V = 16, where HBM bounds and a K-block's conversion takes longer than its
// share of the stream (8B-class layer, 16 vectors: 46.4 us; two groups 51.8).
template <int V>
struct GTile {
    static constexpr int kBV = V;
    static constexpr int kBN = 4 * V;                      // MMA N (digit rows)
    static constexpr int kBTile = kBN * kBK * 2;           // digit bytes per K-block (pair)
    static constexpr int kBHalf = kBTile / 2;              // one CTA's half
    static constexpr int kGroups = V == 64 ? 2 : 4;        // converter groups of four warps = K-blocks of a stage
    static constexpr int kConvWarps = 4 * kGroups;
    static constexpr int kThreads = 32 * (kConvWarps + 8 + 3);
    static constexpr int kStages = 4;                      // of the digit operand, in shared memory
    static constexpr int kAStages = V == 64 ? 2 : 3;       // of M, in TMEM
    static constexpr int kRaw = V == 64 ? 12 : 20;         // K-blocks of int8 M in flight
    static constexpr int kStageBytes = kGroups * kBHalf;
    static constexpr int kRawOff = kStages * kStageBytes;
    static constexpr int kSmem = kRawOff + kRaw * kRawTile + 1024;  // + alignment slack
    static constexpr int kParts = V == 64 ? 2 : 1;         // accumulators a tile is split over
    static constexpr int kPartN = kBN / kParts;            // digit rows (MMA N) of a part
    static constexpr int kPartVecs = V / kParts;           // vectors of a part
    static constexpr int kHalfVecs = kPartVecs / 2;        // of them in one CTA's half of the digit rows
    static constexpr int kAccs = kParts + 1;               // accumulators in TMEM
    static constexpr int kACol = kAccs * kPartN;           // first TMEM column of M
    static constexpr int kAStageCols = kGroups * kBK / 2;  // two fp16 a column
    static constexpr int kTmemCols = 512;
    static constexpr int kVecs = V / 2;                    // vectors per epilogue thread
    static constexpr uint32_t kIdesc = (1u << 4) | ((uint32_t)(kPartN >> 3) << 17) | ((uint32_t)(2 * kBM >> 4) << 24);
    static_assert(kSmem <= 231424, "shared memory per CTA, beside the barriers");
    static_assert(kACol + kAStages * kAStageCols <= kTmemCols, "TMEM allocation");
    static_assert(kAStages <= kStages, "a stage of M is free before its barrier comes round");
};

// First digit row of vector vl in a tile: part by part and CTA by CTA, so that
// a part holds consecutive vectors of the tile.
template <int V>
__device__ __forceinline__ uint32_t tile_row(int vl) {
    using T = GTile<V>;
    const int h = vl / T::kHalfVecs;  // 2 part + CTA
    return (uint32_t)((h & 1) * (T::kBN / 2) + (h >> 1) * (T::kPartN / 2) + 4 * (vl % T::kHalfVecs));
}

// A from TMEM: lane = row, a 32-bit column holds two fp16 of K.
template <uint32_t IDESC>
__device__ __forceinline__ void mma_pair_ta(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(tmem_d),
        "r"(tmem_a), "l"(bdesc), "r"(IDESC), "r"(accumulate)
        : "memory");
}
struct GroupJob {
    const uint8_t *D;         // digit tiles: nvt x nkb blocks of GTile<V>::kBTile bytes
    uint32_t *Y;              // B x m, written directly when split == 1
    unsigned long long *acc;  // B x m partial sums when split > 1
    int m, K, B, nkb, nvt, mp, split, per, item0;
    const uint32_t *Xhat;     // for the digit-tile kernel
    unsigned dblk0, fblk0;    // first block of the job in the digit-tile and split-finish grids
};
struct GroupArgs {
    CUtensorMap map[kMaxGroupJobs];  // M of each job as a K x m tensor of bytes
    GroupJob job[kMaxGroupJobs];
    int njobs, total_items;
    uint4 *acc;               // the split jobs' partial sums, one after the other
    size_t acc_chunks;        // 16-byte chunks of them
    unsigned zero0, zeros;    // blocks of the digit-tile grid that clear them
};

struct Item {
    int j, p, v, kb0, nblk;
};
__device__ __forceinline__ Item group_item(const GroupArgs &a, int idx) {
    int j = 0;
    while (j + 1 < a.njobs && idx >= a.job[j + 1].item0) ++j;
    const GroupJob &g = a.job[j];
    int t = idx - g.item0;
    const int per_p = g.split * g.nvt;
    Item it;
    it.j = j;
    it.p = t / per_p;
    t -= it.p * per_p;
    const int s = t / g.nvt;
    it.v = t - s * g.nvt;
    it.kb0 = s * g.per;
    it.nblk = min(g.nkb, it.kb0 + g.per) - it.kb0;
    return it;
}
// Parts of an item's vector tile that hold vectors.  A tile of up to 32 of them
// is one part: half the MMAs, digits and accumulators (an 8B-class layer for 32
// vectors 71.9 -> 58.0 us, for 96 134.7 -> 118; a 70B-class one for 160 722 ->
// 668).
template <int V>
__device__ __forceinline__ int item_parts(const GroupJob &g, const Item &it) {
    return GTile<V>::kParts == 2 && g.B - it.v * V > GTile<V>::kPartVecs ? 2 : 1;
}
// The r-th item of pair c among C pairs (snake order); -1 past the end.
__device__ __forceinline__ int group_item_index(int r, int c, int C, int total) {
    const int idx = r * C + ((r & 1) ? C - 1 - c : c);
    return idx < total ? idx : -1;
}

// Digit tiles of every job (as k_digit_tiles; job j has the blocks from
// dblk0), and zeroed partial sums of the split jobs (the blocks from zero0).
template <int V>
__global__ void __launch_bounds__(256) k_digit_tiles_grouped(const __grid_constant__ GroupArgs args) {
    using T = GTile<V>;
    // x_hat comes from the kernel before, which may also still use the scratch.
    // Only then may the product start: it reads M without a wait of its own,
    // and the kernel before may be the one that writes M.
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (blockIdx.x >= args.zero0) {
        for (size_t i = (size_t)(blockIdx.x - args.zero0) * 256 + threadIdx.x; i < args.acc_chunks;
             i += (size_t)args.zeros * 256)
            args.acc[i] = make_uint4(0u, 0u, 0u, 0u);
        return;
    }
    int j = 0;
    while (j + 1 < args.njobs && blockIdx.x >= args.job[j + 1].dblk0) ++j;
    const GroupJob &g = args.job[j];
    const size_t gid = (size_t)(blockIdx.x - g.dblk0) * 256 + threadIdx.x;
    const size_t per_vec = (size_t)g.nkb * 8;
    const size_t total = (size_t)g.nvt * T::kBV * per_vec;
    if (gid >= total) return;
    const int v = (int)(gid / per_vec);
    if (v / T::kPartVecs * T::kPartVecs >= g.B) return;  // a part without vectors is not read
    const int grp = (int)(gid % per_vec);
    const int kb = grp >> 3, chunk = grp & 7;
    const int k0 = kb * kBK + chunk * 8;
    // u = centred x_hat + 0x80808080: byte l of u is digit l plus 128 (the
    // signed base-256 digits of limb_split, since 128 (1 + 2^8 + 2^16 + 2^24)
    // added to sum_l 2^(8l) d_l carries nowhere), and the fp16 pattern
    // 0x6400 | (d + 128) is 1024 + d + 128, so one byte permute and one packed
    // add give two digits as exact fp16 values.  K is a multiple of 16 here.
    uint32_t u[8];
    if (v < g.B && k0 < g.K) {
        const uint4 *src = reinterpret_cast<const uint4 *>(g.Xhat + (size_t)v * g.K + k0);
        const uint4 a = src[0], b = src[1];
        const uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = (x[e] > kHalfQ ? x[e] - kQ : x[e]) + 0x80808080u;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = 0x80808080u;  // digits 0
    }
    const int nt = v / T::kBV, vl = v % T::kBV;
    uint8_t *blk = const_cast<uint8_t *>(g.D) + ((size_t)nt * g.nkb + kb) * T::kBTile;
    const __half2 off = __halves2half2(__ushort_as_half(0xE480u), __ushort_as_half(0xE480u));  // -1152
#pragma unroll
    for (int l = 0; l < 4; ++l) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t t = __byte_perm(u[2 * e], u[2 * e + 1], (uint32_t)(l | ((4 + l) << 4)));
            const uint32_t h = __byte_perm(t, 0x64646464u, 0x5140);
            const __half2 d = __hadd2(*reinterpret_cast<const __half2 *>(&h), off);
            w[e] = *reinterpret_cast<const uint32_t *>(&d);
        }
        *reinterpret_cast<uint4 *>(blk + sw128_off(tile_row<V>(vl) + l, chunk)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Y = acc mod q for the split jobs (job j has the blocks from fblk0, four
// outputs per thread).
constexpr int kFinishPer = 4;
__global__ void __launch_bounds__(256) k_split_finish(const __grid_constant__ GroupArgs args) {
    int j = 0;
    while (j + 1 < args.njobs && blockIdx.x >= args.job[j + 1].fblk0) ++j;
    const GroupJob &g = args.job[j];
    const size_t n = (size_t)g.B * g.m, i0 = (size_t)(blockIdx.x - g.fblk0) * (256 * kFinishPer) + threadIdx.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    unsigned long long v[kFinishPer];
#pragma unroll
    for (int u = 0; u < kFinishPer; ++u) v[u] = i0 + 256 * u < n ? g.acc[i0 + 256 * u] : 0ull;
#pragma unroll
    for (int u = 0; u < kFinishPer; ++u)
        if (i0 + 256 * u < n) g.Y[i0 + 256 * u] = fred(v[u]);
}

template <int V>
__global__ void __launch_bounds__(GTile<V>::kThreads, 1)
    k_batched_grouped(const __grid_constant__ GroupArgs args, uint32_t *__restrict__ err, int skip_report,
                      uint64_t wait_ns) {
    using T = GTile<V>;
    constexpr int kGStageBlocks = T::kGroups, kConvW = T::kConvWarps;
    constexpr int kGStages = T::kStages, kGRaw = T::kRaw, kGStageBytes = T::kStageBytes, kGRawOff = T::kRawOff;
    constexpr int kBHalfG = T::kBHalf, kBTileG = T::kBTile, kBVG = T::kBV;
    constexpr int kLoadW = kConvW + 8, kMmaW = kConvW + 9, kWLoadW = kConvW + 10;
    constexpr int kParts = T::kParts, kPartN = T::kPartN, kPartVecs = T::kPartVecs, kAccs = T::kAccs;
    static_assert(kChunkBlocks / kParts % kGStageBlocks == 0, "chunks end on stage boundaries");
    cg::cluster_group cluster = cg::this_cluster();
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full[kGStages], empty_bar[kGStages];
    __shared__ __align__(8) uint64_t acc_full[kAccs], acc_empty[kAccs], mma_done;
    __shared__ __align__(8) uint64_t raw_full[kGRaw], raw_empty[kGRaw];
    __shared__ uint32_t s_tmem;

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(kFull, tid >> 5, 0);  // uniform, so that the roles' operands are
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - smem_addr(smem_raw));
    const uint32_t half = cluster.block_rank() & 1u;  // 0: the even CTA, which issues the MMAs
    const uint16_t pair_mask = 3u;
    const int c = (int)(blockIdx.x >> 1), C = (int)(gridDim.x >> 1);
    const int total = args.total_items;

    // k_split_finish may be put in place beside this kernel; it waits for it
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) {
        for (int s = 0; s < kGStages; ++s) {
            // the digit copies' arrival and, in the even CTA, the odd CTA's
            // report of its own and every converter warp of both CTAs
            mbar_init(&full[s], half == 0 ? 2 * kConvW + 2 : 1);
            mbar_init(&empty_bar[s], 1);
        }
        for (int b = 0; b < kAccs; ++b) {
            mbar_init(&acc_full[b], 1);
            mbar_init(&acc_empty[b], 2 * kEpiThreads / 32);
        }
        mbar_init(&mma_done, 1);
        for (int r = 0; r < kGRaw; ++r) {
            mbar_init(&raw_full[r], 1);
            mbar_init(&raw_empty[r], 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMmaW) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         smem_addr(&s_tmem)), "n"(T::kTmemCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    tc_fence_before();
    cluster.sync();
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    if (warp < kConvW) {
        // ------------------------------------------------ converters: group j fills block j of each stage
        const int grp = warp >> 2;
        const int row = tid & 127;  // = the TMEM lane
        const uint32_t full_leader = cluster_addr(&full[0], 0);
        const uint32_t ta = tmem + ((uint32_t)(row & 96) << 16) + (uint32_t)(T::kACol + grp * (kBK / 2));
        uint32_t gs = 0, gb = 0;
        bool ok = true;
        for (int r = 0; ok; ++r) {
            const int idx = group_item_index(r, c, C, total);
            if (idx < 0) break;
            const Item it = group_item(args, idx);
            for (int b0 = 0; b0 < it.nblk; b0 += kGStageBlocks, ++gs) {
                const int nb = min(kGStageBlocks, it.nblk - b0);
                const uint32_t rb = gb + (uint32_t)grp;
                gb += (uint32_t)nb;
                uint32_t o[kBK / 2];
                // an item's last stage may be short of blocks: the rest only arrive
                if (grp < nb) {
                    const int rs = rb % kGRaw;
                    if (!mbar_wait_warp(&raw_full[rs], (rb / kGRaw) & 1u, err, wait_ns)) {
                        ok = false;
                        break;
                    }
                    // rows of 64 bytes, 64-byte swizzle: eight lanes' chunks lie in distinct banks
                    const uint8_t *raw = smem + kGRawOff + rs * kRawTile + row * kBK;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const uint4 w = *reinterpret_cast<const uint4 *>(raw + ((q ^ ((row >> 1) & 3)) << 4));
                        i8x4_to_f16x4(w.x, o[8 * q], o[8 * q + 1]);
                        i8x4_to_f16x4(w.y, o[8 * q + 2], o[8 * q + 3]);
                        i8x4_to_f16x4(w.z, o[8 * q + 4], o[8 * q + 5]);
                        i8x4_to_f16x4(w.w, o[8 * q + 6], o[8 * q + 7]);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&raw_empty[rs]);
                }
                // the MMAs that read this stage of TMEM are done
                const uint32_t gp = gs - (uint32_t)T::kAStages;
                if (gs >= (uint32_t)T::kAStages &&
                    !mbar_wait_warp(&empty_bar[gp % kGStages], (gp / kGStages) & 1u, err, wait_ns)) {
                    ok = false;
                    break;
                }
                if (grp < nb) {
                    tc_fence_after();
                    tmem_st32(ta + (gs % (uint32_t)T::kAStages) * (uint32_t)T::kAStageCols, o);
                    tc_fence_before();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(full_leader + 8u * (gs % kGStages));
            }
        }
    } else if (warp < kConvW + 8) {
        // ------------------------------------------------ epilogue: TMEM -> mod-q sums -> Y
        const int q = warp & 3;
        const int grp = (warp - kConvW) >> 2;
        const uint32_t acc_empty_leader = cluster_addr(&acc_empty[0], 0);
        uint32_t ev = 0;  // accumulators read
        bool ok = true;
        for (int r = 0; ok; ++r) {
            const int idx = group_item_index(r, c, C, total);
            if (idx < 0) break;
            const Item it = group_item(args, idx);
            const GroupJob &job = args.job[it.j];
            uint32_t run[T::kVecs];
#pragma unroll
            for (int v = 0; v < T::kVecs; ++v) run[v] = 0u;
            auto part = [&](uint32_t *sum) {  // the next accumulator, into a part's sums
                const uint32_t a = ev % kAccs;
                if (!mbar_wait_warp(&acc_full[a], (ev / kAccs) & 1u, err, wait_ns)) {
                    ok = false;
                    return;
                }
                tc_fence_after();
#pragma unroll
                for (int j = 0; j < kPartN / 64; ++j) {
                    uint32_t rr[32];
                    tmem_ld32(tmem + ((uint32_t)(32 * q) << 16) + a * kPartN + (uint32_t)((kPartN / 2) * grp + 32 * j),
                              rr);
#pragma unroll
                    for (int v = 0; v < 8; ++v) {
                        sum[8 * j + v] = fadd(sum[8 * j + v],
                                              digits_redc(__float2int_rn(__uint_as_float(rr[4 * v])),
                                                          __float2int_rn(__uint_as_float(rr[4 * v + 1])),
                                                          __float2int_rn(__uint_as_float(rr[4 * v + 2])),
                                                          __float2int_rn(__uint_as_float(rr[4 * v + 3]))));
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(acc_empty_leader + 8u * a);
                ++ev;
            };
            const int np = item_parts<V>(job, it), seg = kChunkBlocks / np;
            const int nev = (it.nblk + seg - 1) / seg + np - 1;
            for (int i = 0; i < nev && ok; i += np) {
                part(run);
                if (np == 2 && ok && i + 1 < nev) part(run + (kParts - 1) * T::kHalfVecs);
            }
            if (!ok) break;
            const int row = it.p * (2 * kBM) + (int)half * kBM + 32 * q + lane;
            if (row < job.m) {
#pragma unroll
                for (int v = 0; v < T::kVecs; ++v) {
                    const int b = it.v * kBVG + v / T::kHalfVecs * kPartVecs + T::kHalfVecs * grp + v % T::kHalfVecs;
                    if (b < job.B) {
                        const uint32_t val = fmul_mont(run[v], kR2);
                        const size_t o = (size_t)b * job.m + row;
                        if (job.split > 1)
                            atomicAdd(job.acc + o, (unsigned long long)val);
                        else
                            job.Y[o] = val;
                    }
                }
            }
        }
    } else if (warp == kLoadW) {
        // ------------------------------------------------ this CTA's half of the digit operand
        // the digit tiles come from the kernel launched just before this one
        asm volatile("griddepcontrol.wait;" ::: "memory");
        uint32_t gs = 0;
        bool ok = true;
        for (int r = 0; ok; ++r) {
            const int idx = group_item_index(r, c, C, total);
            if (idx < 0) break;
            const Item it = group_item(args, idx);
            const GroupJob &job = args.job[it.j];
            const uint8_t *src = job.D + ((size_t)it.v * job.nkb + it.kb0) * kBTileG + (size_t)half * kBHalfG;
            const uint32_t bytes = (uint32_t)(kBHalfG / kParts * item_parts<V>(job, it));
            for (int b0 = 0; b0 < it.nblk; b0 += kGStageBlocks, ++gs) {
                const int nb = min(kGStageBlocks, it.nblk - b0);
                const int s = gs % kGStages;
                if (!mbar_wait_warp(&empty_bar[s], ((gs / kGStages) & 1u) ^ 1u, err, wait_ns)) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    mbar_arrive_tx(&full[s], (uint32_t)nb * bytes);
                    uint8_t *dst = smem + s * kGStageBytes;
#pragma unroll
                    for (int j = 0; j < kGStageBlocks; ++j)
                        if (j < nb) bulk_g2s(dst + j * kBHalfG, src + (size_t)(b0 + j) * kBTileG, bytes, &full[s]);
                }
                __syncwarp();
            }
        }
        // copies in flight complete before the CTA may exit
        for (uint32_t i = gs > (uint32_t)kGStages ? gs - kGStages : 0u; i < gs; ++i)
            mbar_wait_warp(&full[i % kGStages], (i / kGStages) & 1u, err, wait_ns);
    } else if (warp == kWLoadW) {
        // ------------------------------------------------ raw int8 tiles of M by TMA
        uint32_t gb = 0;
        bool ok = true;
        for (int r = 0; ok; ++r) {
            const int idx = group_item_index(r, c, C, total);
            if (idx < 0) break;
            const Item it = group_item(args, idx);
            const int m0 = it.p * (2 * kBM) + (int)half * kBM;
            const CUtensorMap *map = &args.map[it.j];
            for (int i = 0; i < it.nblk; ++i, ++gb) {
                const int rs = gb % kGRaw;
                if (!mbar_wait_warp(&raw_empty[rs], ((gb / kGRaw) & 1u) ^ 1u, err, wait_ns)) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    mbar_arrive_tx(&raw_full[rs], kRawTile);
                    tma_load_2d(smem + kGRawOff + rs * kRawTile, map, (it.kb0 + i) * kBK, m0, &raw_full[rs]);
                }
                __syncwarp();
            }
        }
        for (uint32_t i = gb > (uint32_t)kGRaw ? gb - kGRaw : 0u; i < gb; ++i)
            mbar_wait_warp(&raw_full[i % kGRaw], (i / kGRaw) & 1u, err, wait_ns);
    } else if (half == 0) {
        // ------------------------------------------------ MMA issuer (even CTA)
        {
            uint32_t gs = 0, ev = 0;  // stages, accumulators finished
            bool ok = true;
            // Accumulators are opened, finished and read in one order, round the
            // kAccs of them.  A segment ends one: of two parts the
            // older, whose chunk began a segment earlier (part 0's first chunk is
            // one segment, so no chunk is longer than kChunkBlocks); the younger
            // opens with the segment.  An item's end finishes both.
            // issue: the MMAs of a stage for one part, into accumulator e
            auto issue = [&](uint32_t e, int part, int nb, bool first) {
                if (first) {
                    if (!mbar_wait_warp(&acc_empty[e % kAccs], ((e / kAccs) & 1u) ^ 1u, err, wait_ns)) return false;
                    tc_fence_after();
                }
                const uint32_t d = tmem + (e % kAccs) * kPartN;
                const uint32_t a = tmem + (uint32_t)T::kACol + (gs % (uint32_t)T::kAStages) * (uint32_t)T::kAStageCols;
                const uint64_t bd =
                    sw128_desc(base) + (((gs % kGStages) * kGStageBytes + part * (kPartN / 2) * 2 * kBK) >> 4);
                if (elect_one()) {
                    mma_pair_ta<T::kIdesc>(d, a, bd, first ? 0u : 1u);
#pragma unroll
                    for (int k = 1; k < kBK / 16; ++k) mma_pair_ta<T::kIdesc>(d, a + 8u * k, bd + 2u * k, 1u);
#pragma unroll
                    for (int j = 1; j < kGStageBlocks; ++j)
                        if (j < nb) {
#pragma unroll
                            for (int k = 0; k < kBK / 16; ++k)
                                mma_pair_ta<T::kIdesc>(d, a + (uint32_t)(j * (kBK / 2) + 8 * k),
                                                       bd + (uint32_t)(j * (kBHalfG >> 4) + 2 * k), 1u);
                        }
                }
                __syncwarp();
                return true;
            };
            for (int r = 0; ok; ++r) {
                const int idx = group_item_index(r, c, C, total);
                if (idx < 0) break;
                const Item it = group_item(args, idx);
                const int np = item_parts<V>(args.job[it.j], it), seg = kChunkBlocks / np;
                const int nseg = (it.nblk + seg - 1) / seg;
                for (int sg = 0; sg < nseg && ok; ++sg, ++ev) {
                    const int b_first = sg * seg, b_end = min(it.nblk, b_first + seg);
                    const int older = np == 2 ? sg & 1 : 0;  // the part that ends with this segment
                    for (int b0 = b_first; b0 < b_end; b0 += kGStageBlocks, ++gs) {
                        const int nb = min(kGStageBlocks, b_end - b0);
                        if (!mbar_wait_warp(&full[gs % kGStages], (gs / kGStages) & 1u, err, wait_ns)) {
                            ok = false;
                            break;
                        }
                        tc_fence_after();
                        if (!issue(ev, older, nb, b0 == (np == 2 ? 0 : b_first))) {
                            ok = false;
                            break;
                        }
                        if (b0 + kGStageBlocks >= b_end) warp_commit_pair(&acc_full[ev % kAccs], pair_mask);
                        if (np == 2 && !issue(ev + 1, 1 - older, nb, b0 == b_first)) {
                            ok = false;
                            break;
                        }
                        warp_commit_pair(&empty_bar[gs % kGStages], pair_mask);
                    }
                }
                if (np == 2) {
                    if (ok) warp_commit_pair(&acc_full[ev % kAccs], pair_mask);
                    ++ev;
                }
            }
            warp_commit_pair(&mma_done, (uint16_t)1u);
            mbar_wait_warp(&mma_done, 0, err, wait_ns);
        }
    } else {
        // ------------------------------------------------ stage relay (odd CTA)
        if (lane == 0) {
            const uint32_t full_leader = cluster_addr(&full[0], 0);
            uint32_t gs = 0;
            bool ok = true;
            for (int r = 0; ok; ++r) {
                const int idx = group_item_index(r, c, C, total);
                if (idx < 0) break;
                const Item it = group_item(args, idx);
                for (int b0 = 0; b0 < it.nblk; b0 += kGStageBlocks, ++gs) {
                    const int s = gs % kGStages;
                    if (!mbar_wait(&full[s], (gs / kGStages) & 1u, err, wait_ns)) {
                        ok = false;
                        break;
                    }
                    // a failure-path test withholds one report (off: skip_report < 0)
                    if ((int)gs == skip_report) continue;
                    mbar_arrive_cluster(full_leader + 8u * (uint32_t)s);
                }
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    cluster.sync();  // the peer is done too: no MMA reads this CTA's memory any more
    if (warp == kMmaW) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(T::kTmemCols));
    }
}

// A job of the grouped launch as the host plans it.
struct PlanJob {
    int src;  // index in the caller's list
    int m, K, B, nkb, nvt, mp, split, per, items;
};

// Blocks per item for a target item size T (in K-blocks).
void plan_splits(std::vector<PlanJob> &jobs, int T) {
    for (PlanJob &j : jobs) {
        int s = (j.nkb + T - 1) / T;
        s = s < 1 ? 1 : (s > kMaxSplit ? kMaxSplit : s);
        j.per = (j.nkb + s - 1) / s;
        j.split = (j.nkb + j.per - 1) / j.per;
        j.items = j.mp * j.split * j.nvt;
    }
}

// Estimated makespan (K-blocks plus a per-item overhead) of the snake
// assignment of the longest-first item list over C pairs.  An overhead of 6
// and 3 for a split item (3 and 1 cut items too short once the K-blocks got
// faster: layers of 3072, 768, 8192 for 64 vectors 52.4 -> 44.6 us, for 128
// 87.4 -> 76.6; 8 and 2, 12 and 2: the same).
double plan_makespan(const std::vector<PlanJob> &jobs, int C) {
    std::vector<double> load(C, 0.0);
    int idx = 0;
    for (const PlanJob &j : jobs) {
        for (int p = 0; p < j.mp; ++p)
            for (int s = 0; s < j.split; ++s) {
                const int nb = std::min(j.nkb, (s + 1) * j.per) - s * j.per;
                for (int v = 0; v < j.nvt; ++v, ++idx) {
                    const int r = idx / C, cc = idx % C;
                    load[(r & 1) ? C - 1 - cc : cc] += nb + 6.0 + (j.split > 1 ? 3.0 : 0.0);
                }
            }
    }
    return *std::max_element(load.begin(), load.end());
}

}  // namespace

bool batched_grouped_eligible(const int8_t *W, const uint32_t *Xhat, int m, int K, int B) {
    return m >= 1 && B >= 1 && K >= 1 && K % 16 == 0 &&
           ((reinterpret_cast<uintptr_t>(W) | reinterpret_cast<uintptr_t>(Xhat)) & 15u) == 0;
}

template <int V>
cudaError_t launch_grouped_v(const BatchJob *jobs, int count, uint32_t *err, cudaStream_t s, bool ready_only) {
    using T = GTile<V>;
    for (int a = 0; a < count; a += kMaxGroupJobs) {
        const int n = std::min(count - a, kMaxGroupJobs);
        std::vector<PlanJob> plan;
        for (int i = 0; i < n; ++i) {
            const BatchJob &b = jobs[a + i];
            PlanJob p{};
            p.src = a + i;
            p.m = b.m;
            p.K = b.K;
            p.B = b.B;
            p.nkb = (b.K + kBK - 1) / kBK;
            p.nvt = (b.B + T::kBV - 1) / T::kBV;
            p.mp = (b.m + 2 * kBM - 1) / (2 * kBM);

            plan.push_back(p);
        }
        const cudaError_t attr =
            func_attr((const void *)k_batched_grouped<V>, cudaFuncAttributeMaxDynamicSharedMemorySize, T::kSmem);
        if (attr != cudaSuccess) return attr;
        const int cap = resident_clusters((const void *)k_batched_grouped<V>, 1);
        // the target item size with the smallest estimated makespan
        static const int kTargets[] = {8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256, 384, 512, 1 << 20};
        double best = 1e300;
        int best_t = 1 << 20, best_c = cap;
        for (int T : kTargets) {
            plan_splits(plan, T);
            std::sort(plan.begin(), plan.end(), [](const PlanJob &x, const PlanJob &y) {
                return x.per != y.per ? x.per > y.per : x.src < y.src;
            });
            int items = 0;
            for (const PlanJob &j : plan) items += j.items;
            const int C = std::min(cap, items);
            const double ms = plan_makespan(plan, C);
            if (ms < best - 1e-9) {
                best = ms;
                best_t = T;
                best_c = C;
            }
        }
        plan_splits(plan, best_t);
        std::sort(plan.begin(), plan.end(), [](const PlanJob &x, const PlanJob &y) {
            return x.per != y.per ? x.per > y.per : x.src < y.src;
        });
        // scratch: digit tiles of every job, then the split jobs' partial sums
        size_t dbytes = 0, abytes = 0;
        for (const PlanJob &j : plan) {
            dbytes += (size_t)j.nvt * j.nkb * T::kBTile;
            if (j.split > 1) abytes += (size_t)j.B * j.m * 8;
        }
        abytes = (abytes + 15) & ~(size_t)15;
        void *buf = nullptr;
        if (ready_only && !stream_scratch_ready(kScratchDigits, dbytes + abytes, s)) return cudaErrorNotReady;
        cudaError_t e = stream_scratch(kScratchDigits, dbytes + abytes, s, &buf);
        if (e != cudaSuccess) return e;
        PFN_cuTensorMapEncodeTiled_v12000 encode = tensor_map_encoder();
        if (!encode) return cudaErrorNotSupported;
        GroupArgs args;
        memset(&args, 0, sizeof(args));
        uint8_t *dp = static_cast<uint8_t *>(buf);
        unsigned long long *ap = reinterpret_cast<unsigned long long *>(dp + dbytes);
        int item0 = 0;
        unsigned dblk = 0, fblk = 0;
        for (int i = 0; i < (int)plan.size(); ++i) {
            const PlanJob &p = plan[i];
            const BatchJob &b = jobs[p.src];
            GroupJob &g = args.job[i];
            g.D = dp;
            dp += (size_t)p.nvt * p.nkb * T::kBTile;
            g.Y = b.Yhat;
            g.acc = nullptr;
            if (p.split > 1) {
                g.acc = ap;
                ap += (size_t)p.B * p.m;
            }
            g.m = p.m;
            g.K = p.K;
            g.B = p.B;
            g.nkb = p.nkb;
            g.nvt = p.nvt;
            g.mp = p.mp;
            g.split = p.split;
            g.per = p.per;
            g.item0 = item0;
            g.Xhat = b.Xhat;
            item0 += p.items;
            g.dblk0 = dblk;
            dblk += (unsigned)(((size_t)p.nvt * T::kBV * p.nkb * 8 + 255) / 256);
            g.fblk0 = fblk;
            if (p.split > 1) fblk += (unsigned)(((size_t)p.B * p.m + 256 * kFinishPer - 1) / (256 * kFinishPer));
            const cuuint64_t gdim[2] = {(cuuint64_t)p.K, (cuuint64_t)p.m};
            const cuuint64_t gstride[1] = {(cuuint64_t)p.K};
            const cuuint32_t box[2] = {(cuuint32_t)kBK, (cuuint32_t)kBM};
            const cuuint32_t estride[2] = {1, 1};
            if (encode(&args.map[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t *>(b.W), gdim, gstride,
                       box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B,
                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
                return cudaErrorInvalidValue;
        }
        args.njobs = (int)plan.size();
        args.total_items = item0;
        if (item0 == 0) continue;
        // digit tiles, and 1 KiB or more of the partial sums per further block
        args.acc = reinterpret_cast<uint4 *>(static_cast<uint8_t *>(buf) + dbytes);
        args.acc_chunks = abytes / 16;
        args.zero0 = dblk;
        args.zeros = (unsigned)std::min<size_t>(1024, (args.acc_chunks + 255) / 256);
        cudaLaunchAttribute pdl[1];
        pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        pdl[0].val.programmaticStreamSerializationAllowed = 1;
        cudaLaunchConfig_t dcfg = {};
        dcfg.gridDim = dim3(dblk + args.zeros, 1, 1);
        dcfg.blockDim = dim3(256, 1, 1);
        dcfg.stream = s;
        dcfg.attrs = pdl;
        dcfg.numAttrs = 1;
        e = counted_launch(cudaLaunchKernelEx(&dcfg, k_digit_tiles_grouped<V>, args));
        if (e != cudaSuccess) return e;
        const int C = std::min(best_c, item0);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(2 * C, 1, 1);
        cfg.blockDim = dim3(T::kThreads, 1, 1);
        cfg.dynamicSmemBytes = T::kSmem;
        cfg.stream = s;
        cudaLaunchAttribute lattr[2];
        lattr[0].id = cudaLaunchAttributeClusterDimension;
        lattr[0].val.clusterDim.x = 2;
        lattr[0].val.clusterDim.y = 1;
        lattr[0].val.clusterDim.z = 1;
        lattr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        lattr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = lattr;
        cfg.numAttrs = 2;
        const DebugWait dbg = debug_wait();
        const int skip_report = dbg.site == PVMVMD_DEBUG_WAIT_PRODUCT ? (int)dbg.index : -1;
        const uint64_t wait_ns = dbg.site == PVMVMD_DEBUG_WAIT_PRODUCT ? dbg.limit : kWaitNs;
        e = counted_launch(cudaLaunchKernelEx(&cfg, k_batched_grouped<V>, args, err, skip_report, wait_ns));
        if (e != cudaSuccess) return e;
        if (fblk) {
            // jobs without splits before a split one share its first block
            // index; the last such job is the one the kernel finds
            cudaLaunchConfig_t fcfg = {};
            fcfg.gridDim = dim3(fblk, 1, 1);
            fcfg.blockDim = dim3(256, 1, 1);
            fcfg.stream = s;
            fcfg.attrs = pdl;
            fcfg.numAttrs = 1;
            e = counted_launch(cudaLaunchKernelEx(&fcfg, k_split_finish, args));
            if (e != cudaSuccess) return e;
        }
    }
    return cudaSuccess;
}

cudaError_t launch_batched_grouped(const BatchJob *jobs, int count, uint32_t *err, cudaStream_t s, bool ready_only) {
    // small batches in 16-vector tiles, the rest in 64-vector tiles
    std::vector<BatchJob> narrow, wide;
    for (int i = 0; i < count; ++i) (jobs[i].B <= kNarrowMaxB ? narrow : wide).push_back(jobs[i]);
    cudaError_t e = cudaSuccess;
    if (!wide.empty()) e = launch_grouped_v<64>(wide.data(), (int)wide.size(), err, s, ready_only);
    if (e == cudaSuccess && !narrow.empty()) e = launch_grouped_v<16>(narrow.data(), (int)narrow.size(), err, s, ready_only);
    return e;
}

cudaError_t launch_batched(const int8_t *W, int m, int K, const uint32_t *Xhat, int B,
                           uint32_t *Yhat, uint32_t *err, cudaStream_t s) {
    if (m <= 0 || K <= 0 || B <= 0) return cudaSuccess;
    if (batched_grouped_eligible(W, Xhat, m, K, B)) {
        const BatchJob job{W, Xhat, Yhat, m, K, B};
        return launch_batched_grouped(&job, 1, err, s);
    }
    const int nkb = (K + kBK - 1) / kBK;
    const int nvt = (B + kBV - 1) / kBV;
    void *D = nullptr;
    cudaError_t e = stream_scratch(kScratchDigits, (size_t)nvt * nkb * kBTile, s, &D);
    if (e != cudaSuccess) return e;
    return batched_launch(W, m, K, Xhat, B, Yhat, err, static_cast<uint8_t *>(D), s);
}

}  // namespace pv

// ---------------------------------------------------------------------------
// pvmvmd_server_mvm_noalloc: the batched product with its digit tiles in a
// fixed file-scope device array instead of a buffer the library allocates.
// ---------------------------------------------------------------------------
namespace pv {
namespace {

constexpr size_t kNoAllocBytes = PVMVMD_NOALLOC_SCRATCH_BYTES;
static __device__ __align__(256) uint8_t g_noalloc_tiles[kNoAllocBytes];

// Device address of g_noalloc_tiles on the current device.  Host code may
// not use the symbol itself (its host-side name is only a stand-in), so it is
// looked up once per device, with that device current.  Under lazy module
// loading the lookup loads this file's module on the device, which is when
// the device reserves the array.
cudaError_t noalloc_tiles(uint8_t **out) {
    static std::mutex mu;
    static uint8_t *addr[64] = {nullptr};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mu);
    if (!addr[dev]) {
        void *p = nullptr;
        e = cudaGetSymbolAddress(&p, g_noalloc_tiles);
        if (e != cudaSuccess) return e;
        addr[dev] = static_cast<uint8_t *>(p);
    }
    *out = addr[dev];
    return cudaSuccess;
}

}  // namespace
}  // namespace pv

extern "C" int pvmvmd_server_mvm_noalloc(const int8_t *W_dev, int m, int K, const uint32_t *Xhat_dev,
                                         int B, uint32_t *Yhat_dev, void *stream) {
    using namespace pv;
    if (!W_dev || !Xhat_dev || !Yhat_dev) return PVMVMD_E_ARG;
    if (m < 1 || K < 1 || K > PVMVMD_MAX_K || B < 1) return PVMVMD_E_SHAPE;
    const int nkb = (K + kBK - 1) / kBK;
    const int nvt = (B + kBV - 1) / kBV;
    const size_t need = (size_t)nvt * nkb * kBTile;
    if (need > kNoAllocBytes) return PVMVMD_E_SHAPE;  // beyond the fixed buffer
    uint8_t *D = nullptr;
    const cudaError_t lookup = noalloc_tiles(&D);
    if (lookup != cudaSuccess) {
        (void)cudaGetLastError();
        // under lazy module loading the lookup is when the array is reserved
        return lookup == cudaErrorMemoryAllocation ? PVMVMD_E_NOMEM : PVMVMD_E_CUDA;
    }
    uint32_t *err = library_error_word();
    if (!err) return PVMVMD_E_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(stream);

    // every byte of the tiles in use is rewritten: nothing left by an
    // earlier call is read
    if (batched_launch(W_dev, m, K, Xhat_dev, B, Yhat_dev, err, D, s) != cudaSuccess) {
        (void)cudaGetLastError();
        return PVMVMD_E_CUDA;
    }
    return PVMVMD_OK;
}
