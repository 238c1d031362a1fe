// Attention of new tokens over a paged cache (pvmvmd_paged_attention): which kernel
// takes which sequences.
#include "attention.h"
#include "kv.cuh"

namespace pv {

// Sequences of at most kFewRows rows per key head, single generated tokens above all,
// go to the kernel that reads K and V as fast as they come, and where no sequence has
// more than kFewWholeKeys keys those of kFewRowsWhole rows (eight tokens of 32 rows over
// themselves 9.6 us on the tensor cores' path, most of it set-up).  The others go to
// the tensor cores.  A call may have both; the host knows the largest number of new
// tokens at most, and which sequence has how many is seen on the device.
cudaError_t launch_attention(const AttendJob &job, const KvView &kv, cudaStream_t s) {
    AttendJob j = job;
    const int G = j.Hq / kv.heads;
    j.few_rows = (int64_t)kv.max_pages * kv.ps.d <= kFewWholeKeys ? kFewRowsWhole : kFewRows;
    const bool one = kv.B == 1;  // which has all the new tokens
    bool few = false, joined = false;
    if (G > j.few_rows)
        j.few_rows = 0;
    else if (!(one && (int64_t)kv.T * G > j.few_rows)) {
        const cudaError_t e = launch_attention_few(j, kv, s);
        if (e != cudaSuccess) return e;
        if (one || j.max_new <= j.few_rows / G) return launch_attention_few_finish(j, kv, s);
        few = true;
    }
    if (j.accumulate) {
        void *p = nullptr;
        const cudaError_t e = stream_scratch(kScratchLse, (size_t)kv.T * j.Hq * sizeof(float), s, &p);
        if (e != cudaSuccess) return e;
        j.lse2 = static_cast<float *>(p);
    }
    // Where there are both, they run beside one another: the chunks beside the few rows,
    // the few rows' join beside the chunks', and else beside the mass.  (104 sequences of
    // 1 to 8 new tokens with mass: XX us a call where XX one after the other.)
    j.beside = few;
    cudaError_t e = launch_attention_chunk(j, kv, s, joined);
    if (e != cudaSuccess) return e;
    j.beside = joined;
    if (few) e = launch_attention_few_finish(j, kv, s);
    if (e != cudaSuccess || !j.accumulate) return e;
    j.beside = few && !joined;
    return launch_attention_mass(j, kv, s);
}

}  // namespace pv
