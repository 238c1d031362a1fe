// The host side of the client's attention (csrc/attention_api.cu) with launches that
// only take time: which of them are under way together, and what a call does where the
// host's memory is at an end.  Driven by test_attention_host.py.
#include <atomic>
#include <chrono>
#include <cstdlib>
#include <new>
#include <thread>

#include <cuda_runtime.h>

// named by device code that is compiled for the host here and never run
static inline unsigned __umulhi(unsigned, unsigned) { return 0; }
static inline unsigned atomicOr(unsigned *, unsigned) { return 0; }
template <typename T> T __ldg(const T *p) { return *p; }
static inline unsigned __funnelshift_l(unsigned, unsigned, unsigned) { return 0; }
static inline unsigned __funnelshift_r(unsigned, unsigned, unsigned) { return 0; }
static inline int max(int a, int b) { return a < b ? b : a; }
static inline int min(int a, int b) { return b < a ? b : a; }

static std::atomic<bool> g_no_memory;
void *operator new(size_t n) {
    void *p = g_no_memory ? nullptr : std::malloc(n ? n : 1);
    if (!p) throw std::bad_alloc();
    return p;
}
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, size_t) noexcept { std::free(p); }

#include "attention_api.cu"
#include "scratch.cu"

namespace {
std::atomic<int> g_in[3], g_all, g_most[3], g_most_all;
void note(std::atomic<int> &now, std::atomic<int> &most) {
    const int n = ++now;
    for (int m = most; n > m && !most.compare_exchange_weak(m, n);) {
    }
}
cudaError_t take_time(cudaStream_t s) {
    const size_t i = reinterpret_cast<size_t>(s);
    note(g_in[i], g_most[i]);
    note(g_all, g_most_all);
    std::this_thread::sleep_for(std::chrono::milliseconds(100));
    --g_in[i];
    --g_all;
    return cudaSuccess;
}
}  // namespace

namespace pv {
cudaError_t launch_rope(const RopeJob &, const KvView *, cudaStream_t) { return cudaSuccess; }
cudaError_t launch_attention(const AttendJob &, const KvView &, cudaStream_t s) { return take_time(s); }
cudaError_t launch_evict(const EvictJob &, const KvView &, cudaStream_t s) { return take_time(s); }
}  // namespace pv

extern "C" {
cudaError_t cudaGetDevice(int *dev) {
    *dev = 0;
    return cudaSuccess;
}
cudaError_t cudaGetLastError(void) { return cudaSuccess; }
cudaError_t cudaMalloc(void **, size_t) { return cudaErrorMemoryAllocation; }
cudaError_t cudaFree(void *) { return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaStreamIsCapturing(cudaStream_t, cudaStreamCaptureStatus *st) {
    *st = cudaStreamCaptureStatusNone;
    return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void *, cudaFuncAttribute, int) { return cudaSuccess; }

void host_reset(void) {
    g_most_all = 0;
    for (std::atomic<int> &m : g_most) m = 0;
}
int host_most(int stream) { return stream < 0 ? g_most_all : g_most[stream]; }

// What a call returns while the host has no memory; 1000: it threw.
int host_without_memory(int what, const pvmvmd_kv_pool *pool, const pvmvmd_kv_batch *batch) {
    void *p = reinterpret_cast<void *>(4096), *s = reinterpret_cast<void *>((size_t)2), *out;
    int status = 1000;
    g_no_memory = true;
    try {
        status = what == 0   ? pvmvmd_paged_attention(pool, batch, 2, p, 64, 64, 1.0f, 1, 0, 0, p, 64, 64, nullptr, s)
                 : what == 1 ? pvmvmd_kv_evict(pool, batch, 8, 2, (int32_t *)p, 4, 4, (int32_t *)p, s)
                 : what == 2 ? (int)pv::stream_scratch(pv::kScratchDigits, 100, (cudaStream_t)s, &out)
                             : (int)pv::func_attr(p, cudaFuncAttributeMaxDynamicSharedMemorySize, 1000);
    } catch (...) {
    }
    g_no_memory = false;
    return status;
}
void host_forget(void) {
    pv::g_bufs.clear();
    pv::g_turns.clear();
}
}
