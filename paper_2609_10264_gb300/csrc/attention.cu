// Attention of new tokens over a paged cache (pvmvmd_paged_attention): which kernel
// takes which sequences.
#include <algorithm>

#include "attention.h"
#include "kv.cuh"

namespace pv {

int64_t seen_keys(const AttendJob &j, const KvView &kv, int align) {
    const int64_t room = (int64_t)kv.max_pages * kv.ps.d;
    return j.window > 0 ? std::min(room, (int64_t)j.window + j.max_new + align - 2) : room;
}
int score_rows(const AttendJob &j, const KvView &kv) {
    return (int)std::min<int64_t>(j.few_rows, ((int64_t)j.max_new * (j.Hq / kv.heads) + 3) / 4 * 4);
}

// Rows per key head (new tokens x query heads of it) up to which a sequence, single
// generated tokens above all, goes to the kernel that reads K and V as fast as they
// come; the others go to the tensor cores' path.
//   64 where no sequence can have more than kFewWholeKeys keys (eight tokens of 32 rows
//   over themselves 9.6 us on the tensor cores' path, most of it set-up);
//   32, two passes over the keys, where that path's set-up or its kernel for the mass
//   costs more: K and V of no more than kFewBytes (24 rows over 6000 keys 25 -> 22 us, 16
//   such over 2000 41 -> 32) or mass (43 -> 33 and 57 -> 44; 64 over 4000 224 -> 214);
//   16 beyond (32 rows over 60000 keys 55 us, in two passes 68; 24 rows of 64 sequences
//   over 4000 121 and 135), and where others have more rows, so that the tensor cores'
//   path runs anyway (five of 19 to 56 rows over 16000 keys 57 us, some of them in two
//   passes 65, with mass 107 and 125).
int few_rows(const AttendJob &j, const KvView &kv) {
    const int64_t room = (int64_t)kv.max_pages * kv.ps.d, seen = j.window > 0 ? (int64_t)j.window + j.max_new : room;
    if (room <= kFewWholeKeys) return kFewRowsWhole;
    const int64_t bytes = 4 * kv.dim * std::min(room, seen) * kv.heads * kv.B;
    const bool all = (int64_t)j.max_new * (j.Hq / kv.heads) <= 2 * kFewRows;
    return all && (j.accumulate || bytes <= kFewBytes) ? 2 * kFewRows : kFewRows;
}

// A call may have sequences for both; the host knows the largest number of new tokens at
// most, and which sequence has how many is seen on the device.
cudaError_t launch_attention(const AttendJob &job, const KvView &kv, cudaStream_t s) {
    AttendJob j = job;
    const int G = j.Hq / kv.heads;
    j.few_rows = few_rows(j, kv);
    bool few = false, joined = false;
    const int64_t most = (int64_t)j.max_new * G;  // rows of a sequence
    // Scores that k_few would keep for the mass.  Their room goes by the table, as the lengths
    // are on the device; beyond kMostScores the tensor cores' path takes all sequences,
    // which forms the scores anew (64 sequences of 8 heads of 8 rows reach that with room for
    // 131072 keys, of which up to 8192 are there: 300 us, just beyond it 494; with room for 2^20,
    // 495, k_few would ask for 17 GB).
    const double scores = (double)sizeof(float) * kv.B * kv.heads * seen_keys(j, kv, kFewMostTile) * score_rows(j, kv);
    if (G > j.few_rows || (kv.B == 1 && most > j.few_rows) || (j.accumulate && scores > kMostScores)) {
        // A single sequence goes there whole, however few of `most` rows the device finds.
        j.few_rows = 0;
    } else {
        const cudaError_t e = launch_attention_few(j, kv, s);
        if (e != cudaSuccess) return e;
        if (most <= j.few_rows) return launch_attention_few_finish(j, kv, s);
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
    // 1 to 8 new tokens with mass: 44 us a call where 65 one after the other.)
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
