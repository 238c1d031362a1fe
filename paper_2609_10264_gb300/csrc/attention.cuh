// What the kernels of the client's attention share.
#pragma once

#include "attention.h"
#include "kv.cuh"
#include "tensor.cuh"

namespace pv {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 16 bytes, or zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void shared_store16(uint32_t dst, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint4 shared_load16(uint32_t src) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(src) : "memory");
    return v;
}
__device__ __forceinline__ void copy4(uint32_t dst, const void *src, bool real) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(real ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// An arrival of this thread's on bar once its copies so far are there (bar counts it).
__device__ __forceinline__ void copy_arrive(uint64_t *bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::
            "r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_addr(bar))
        : "memory");
}
template <int N>
__device__ __forceinline__ void copy_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t pack(float x, float y, __half) {
    const __half2 v = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack(float x, float y, __nv_bfloat16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}


// ---------------------------------------------------------------- pairs of 32-bit values
// (half the instructions of the softmax's multiply-adds and sums)
__device__ __forceinline__ uint64_t pair(float x, float y) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float &x, float &y) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Where a share of work lies among the sequences' works.  By all threads of the CTA.
struct Found {
    int64_t total, before;  // all the work, and that of the sequences before b
    int b;
};
// The sequence that holds position pos(total) of all the work (a negative one: none).
// The work before each sequence, and behind them all of it, goes to `list`, if there.
template <int kThreads, typename Work, typename Pos>
__device__ __forceinline__ Found find(int B, Work work, Pos pos, int64_t *list = nullptr) {
    __shared__ int64_t s_warp[kThreads / 32], s_before;
    __shared__ int s_b;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (B == 1) {
        const int64_t w = work(0), p = pos(w);
        if (list && tid == 0) list[0] = 0, list[1] = w;
        return Found{w, 0, p >= 0 && p < w ? 0 : -1};
    }
    if (B <= 32) {  // every warp by itself, a lane a sequence
        const int64_t w = lane < B ? work(lane) : 0;
        int64_t incl = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t v = __shfl_up_sync(kFull, incl, o);
            if (lane >= o) incl += v;
        }
        const int64_t total = __shfl_sync(kFull, incl, 31), pre = incl - w, p = pos(total);
        if (list && warp == 0 && lane < B) list[lane] = pre;
        if (list && tid == 0) list[B] = total;
        const unsigned at = __ballot_sync(kFull, p >= pre && p < incl);
        const int b = at ? __ffs(at) - 1 : 0;
        return Found{total, __shfl_sync(kFull, pre, b), at ? b : -1};
    }
    const int per = (B + kThreads - 1) / kThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    int64_t sum = 0;
    for (int b = b0; b < b1; ++b) sum += work(b);
    int64_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(kFull, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) s_warp[warp] = incl;
    if (tid == 0) s_before = 0, s_b = -1;
    __syncthreads();
    int64_t total = 0, base = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) base += s_warp[w];
        total += s_warp[w];
    }
    int64_t pre = base + incl - sum;
    if (list) {
        int64_t at = pre;
        for (int b = b0; b < b1; ++b) {
            list[b] = at;
            at += per == 1 ? sum : work(b);
        }
        if (tid == 0) list[B] = total;
    }
    const int64_t p = pos(total);
    if (p >= pre && p < pre + sum && per == 1) {
        s_before = pre, s_b = b0;
    } else if (p >= pre && p < pre + sum) {
        for (int b = b0; b < b1; ++b) {
            const int64_t w = work(b);
            if (p >= pre && p < pre + w) s_before = pre, s_b = b;
            pre += w;
        }
    }
    __syncthreads();
    return Found{total, s_before, s_b};
}

// Launched as soon as the kernel before lets it, which it waits for itself: every
// kernel here begins with `follow`, so that only its launch goes beside the end of the
// one before.  (What the dependents of this one read before their own wait is then
// complete, too.)
template <typename K, typename... A>
cudaError_t launch_cluster(K kern, dim3 grid, int cluster, int threads, size_t smem, cudaStream_t s, const A &...a) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return counted_launch(cudaLaunchKernelEx(&cfg, kern, a...));
}
template <typename K, typename... A>
cudaError_t launch_dependent(K kern, dim3 grid, int threads, size_t smem, cudaStream_t s, const A &...a) {
    return launch_cluster(kern, grid, 1, threads, smem, s, a...);
}
__device__ __forceinline__ void follow(bool beside = false) {
    if (!beside) asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// A kernel that uses nothing of the one before may run beside it: that one is past its
// own wait when this one starts, so what came before it is complete.  This one then ends
// after it, for those that follow (by the first CTA).
__device__ __forceinline__ void end_after(bool beside) {
    if (beside && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0)
        asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ---------------------------------------------------------------- tensor cores
// What the chunk kernels share: CTAs of three warpgroups, two that compute and one of
// which a warp issues MMAs and three copy tiles of 128 rows.
constexpr int kCM = 128;             // rows per tile
constexpr int kCN = 128;             // keys per tile
constexpr int kCThreads = 384;
constexpr int kCLoaders = 3;         // warps 9-11
constexpr int kCSoftRegs = 208, kCOtherRegs = 80;

// The copy of a tile of 128 rows of up to DP 16-bit values by one warp, into the
// 128-byte-swizzled layout: slabs of 64 values, 16 KiB each.
template <int DP>
struct TileCopy {
    static constexpr int kPerRow = DP / 8, kRowsAt = 32 / kPerRow;  // 16-byte chunks, rows per instruction
    int lane, ch, sub;
    bool real;  // this lane's chunk is one of the row's
    __device__ __forceinline__ TileCopy(int lane_, int dim)
        : lane(lane_), ch(lane_ % kPerRow), sub(lane_ / kPerRow), real(lane_ % kPerRow * 8 < dim) {}
    // Rows first .. first + 32 kBlocks - 1.  row(rr, off): whether row rr is there, and
    // its place from src on; else zeros.
    template <int kBlocks = kCM / 32, typename Row>
    __device__ __forceinline__ void copy(uint32_t dst, const char *src, Row row, int first = 0) const {
        int64_t off[kBlocks];
        unsigned there[kBlocks];
#pragma unroll
        for (int x = 0; x < kBlocks; ++x) {
            const bool is = row(first + 32 * x + lane, off[x]);
            if (!is) off[x] = 0;
            there[x] = __ballot_sync(kFull, is);
        }
        src += real ? ch * 16 : 0;
        dst += (uint32_t)(ch >> 3) * (kCM * 128);
        // some places at a time, then their copies, which the compiler keeps in order
        constexpr int kBatch = 4;
#pragma unroll
        for (int u0 = 0; u0 < 32 * kBlocks / kRowsAt; u0 += kBatch) {
            int64_t o[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int rr = (u0 + u) * kRowsAt;
                o[u] = __shfl_sync(kFull, off[rr / 32], (rr + sub) & 31);
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int rr = (u0 + u) * kRowsAt;
                copy16(dst + sw128_off(first + rr + sub, ch & 7), src + o[u], real && (there[rr / 32] >> ((rr + sub) & 31) & 1));
            }
        }
        copy_commit();
    }
    // The 128 keys from key0 on from their pages by the tensor memory accelerator: boxes
    // of `box` keys that lie on one page, dealt out to the lanes; map: (values, slots,
    // heads, pages).  False, and nothing done, where a page is not there.  Behind the
    // sequence's end the rows hold anything.  (The swizzle goes by the address, so boxes of
    // fewer than its eight rows fit too.)
    __device__ __forceinline__ bool fetch(uint32_t dst, const CUtensorMap *map, int box, const KvView &kv, int b, int hk,
                                          int key0, int len, uint64_t *bar) const {
        const int end = max(0, min(kCM, (len - key0 + box - 1) / box * box));  // of the boxes
        int page[kCM / 32], slot[kCM / 32];
        bool there = true;
#pragma unroll
        for (int x = 0; x < kCM / 32; ++x) {
            page[x] = slot[x] = 0;
            const int r = (32 * x + lane) * box;
            if (r < end) there &= kv.place(b, key0 + r, page[x], slot[x]);
        }
        if (!__all_sync(kFull, there)) return false;
        if (lane == 0) mbar_arrive_tx(bar, (uint32_t)(DP / 64 * end * 128));
        __syncwarp();
#pragma unroll
        for (int x = 0; x < kCM / 32; ++x) {
            const int r = (32 * x + lane) * box;
            if (r < end)
#pragma unroll
                for (int s = 0; s < DP / 64; ++s)
                    asm volatile(
                        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, "
                        "%4, %5}], [%6];" ::"r"(dst + s * (kCM * 128) + r * 128),
                        "l"(reinterpret_cast<uint64_t>(map)), "r"(64 * s), "r"(slot[x]), "r"(hk), "r"(page[x]),
                        "r"(smem_addr(bar))
                        : "memory");
        }
        return true;
    }
    // Once it is all there, for the MMAs.
    __device__ __forceinline__ void arrive(uint64_t *bar, int tiles = 1) const {
        copy_wait<0>();
        fence_async_smem();
        __syncwarp();
        for (int t = 0; lane == 0 && t < tiles; ++t) mbar_arrive(bar);
    }
};

template <typename T>
__device__ __forceinline__ constexpr uint32_t chunk_idesc(int n) {
    const uint32_t f = __is_same(T, __half) ? 0u : 1u;
    return (1u << 4) | (f << 7) | (f << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kCM >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar))
                 : "memory");
}
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, float *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
        "%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
          "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]),
          "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]),
          "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld16_async(uint32_t taddr, float *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
          "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }


// Keys per TMA box: the largest power of two, up to a tile, that divides the page size;
// none where that is less than 4, and none where a stride is not one that a tensor map
// can have.  (2048 tokens over 8192 keys, 32 heads of 128, us: boxes of 1 key 612, of 2
// 341, of 4 220, of 8 169, of 64 165; gathered row by row by the loaders 271 in pages of 2,
// 277 of 1.)
constexpr int kLeastBox = 4;
inline int page_box(const KvView &kv) {
    int box = 1;
    while (box < kCN && kv.ps.d % (2 * box) == 0) box *= 2;
    const int64_t most = (int64_t)1 << 40;
    for (int64_t st : {kv.k_slot, kv.k_head, kv.k_page, kv.v_slot, kv.v_head, kv.v_page})
        if (st <= 0 || st >= most) return 0;
    return box >= kLeastBox ? box : 0;
}
// Keys or values as a tensor of (values, slots, heads, pages), for boxes of 64 values
// x `box` slots.
inline cudaError_t page_map(CUtensorMap *map, const KvView &kv, bool values, int type, int box) {
    PFN_cuTensorMapEncodeTiled_v12000 encode = tensor_map_encoder();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t dim[4] = {(cuuint64_t)kv.dim, kv.ps.d, (cuuint64_t)kv.heads, (cuuint64_t)kv.pages};
    const cuuint64_t stride[3] = {(cuuint64_t)(values ? kv.v_slot : kv.k_slot), (cuuint64_t)(values ? kv.v_head : kv.k_head),
                                  (cuuint64_t)(values ? kv.v_page : kv.k_page)};
    const cuuint32_t part[4] = {64, (cuuint32_t)box, 1, 1}, one[4] = {1, 1, 1, 1};
    const CUresult r = encode(map, type == PVMVMD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
                              4, values ? kv.V : kv.K, dim, stride, part, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// New rows as a tensor of (values, heads, tokens), for boxes of a key head's heads and
// as many tokens as make a tile; false where a tile is not whole tokens, or the strides
// are such that a tensor map cannot have them.
inline bool rows_map(CUtensorMap *map, const AttendJob &j, const KvView &kv, int G) {
    PFN_cuTensorMapEncodeTiled_v12000 encode = tensor_map_encoder();
    if (!encode || kCM % G || j.q_token <= 0 || j.q_head <= 0) return false;
    const cuuint64_t dim[3] = {(cuuint64_t)kv.dim, (cuuint64_t)j.Hq, (cuuint64_t)kv.T};
    const cuuint64_t stride[2] = {(cuuint64_t)j.q_head, (cuuint64_t)j.q_token};
    const cuuint32_t part[3] = {64, (cuuint32_t)G, (cuuint32_t)(kCM / G)}, one[3] = {1, 1, 1};
    return encode(map, j.type == PVMVMD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                  const_cast<void *>(j.q), dim, stride, part, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Cache index i of sequence b, of length len: whether it is there, and its place in
// K or V (strides in bytes).  No branch, so that several look-ups run at a time.
__device__ __forceinline__ bool key_place(const KvView &kv, int b, int len, int i, int64_t page_stride,
                                          int64_t slot_stride, int64_t &off) {
    int page, slot;
    const bool is = kv.place(b, max(min(i, len - 1), 0), page, slot) && i < len;
    off = page * page_stride + slot * slot_stride;
    return is;
}

// New rows of sequence b per key head, where they are too many for the kernel of few.
__device__ __forceinline__ int many_rows(const KvView &kv, int few_rows, int G, int b) {
    const int rows = kv.news(b) * G;
    return rows <= few_rows ? 0 : rows;
}

// 1 / L for a row's sum, 0 for one that sees nothing (M its maximum).
__device__ __forceinline__ float inverse(float M, float L) { return M == -INFINITY ? 0.0f : 1.0f / L; }

}  // namespace
}  // namespace pv
