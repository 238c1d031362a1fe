// Attention of new tokens over a paged cache (pvmvmd_paged_attention): which kernel
// takes which sequences.
#include "attention.h"
#include "kv.cuh"

namespace pv {

// Sequences of at most kFewRows rows per key head, single generated tokens above all,
// go to the kernel that reads K and V as fast as they come; the others to the tensor
// cores.  A call may have both; the host knows the largest number of new tokens at
// most, and which sequence has how many is seen on the device.
cudaError_t launch_attention(const AttendJob &job, const KvView &kv, cudaStream_t s) {
    AttendJob j = job;
    const int G = j.Hq / kv.heads;
    const bool one = kv.B == 1;  // which has all the new tokens
    if (G <= kFewRows && !(one && (int64_t)kv.T * G > kFewRows)) {
        const cudaError_t e = launch_attention_few(j, kv, s);
        if (e != cudaSuccess || one || j.max_new <= kFewRows / G) return e;
    }
    if (j.accumulate) {
        void *p = nullptr;
        const cudaError_t e = stream_scratch(kScratchLse, (size_t)kv.T * j.Hq * sizeof(float), s, &p);
        if (e != cudaSuccess) return e;
        j.lse2 = static_cast<float *>(p);
    }
    const cudaError_t e = launch_attention_chunk(j, kv, s);
    return e != cudaSuccess || !j.accumulate ? e : launch_attention_mass(j, kv, s);
}

}  // namespace pv
