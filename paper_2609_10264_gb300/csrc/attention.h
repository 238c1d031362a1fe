// Host-side launchers of the client's attention (internal to the library).
#pragma once

#include "launch.h"

namespace pv {

struct KvView;

// Heads of one tensor: strides in elements.
struct RopePart {
    const void *src;
    void *dst;  // part 0 alone; parts 1 and 2 go to the cache
    int64_t src_token, src_head, dst_token, dst_head;
    int heads;
};
struct RopeJob {
    const uint64_t *turns;
    const int32_t *pos;  // null: cache indexes
    RopePart part[3];    // q (or x), k, v
    int T, dim, rot, interleaved, in_type, out_type;
    float magnitude, scale;
    bool cached;  // parts 1 and 2 are there
};
cudaError_t launch_rope(const RopeJob &j, const KvView *kv, cudaStream_t s);

struct AttendJob {
    const void *q;
    void *out;
    float *lse;                              // may be null
    float *lse2;                             // scratch: -log2 of the rows' sums (see row_sum), may be null
    int64_t q_token, q_head, o_token, o_head;  // bytes
    int Hq, window, type, max_new;           // window 0: none
    int few_rows;                            // see launch_attention_few
    float scale;
    bool causal, accumulate;
    bool beside;  // the kernel before is of the same call, and of other sequences
};
cudaError_t launch_attention(const AttendJob &j, const KvView &kv, cudaStream_t s);
// Of the sequences with at most few_rows new rows per key head (tokens x query heads
// of it); the others are left alone.  Where no sequence has more keys than
// kFewWholeKeys rows are cheap.
constexpr int kFewRows = 16, kFewRowsWhole = 64, kFewWholeKeys = 512;
constexpr int64_t kFewBytes = 192 << 20;
// Bytes of scratch at most for the scores of few rows (see launch_attention) and, as
// long as an item has several splits, for the parts of chunks.
constexpr int64_t kMostScores = (int64_t)2 << 30, kMostParts = (int64_t)1 << 30;
constexpr int kFewMostTile = 256;  // keys per tile of launch_attention_few
// Keys of a sequence, from a boundary of `align` on, that any of its new rows may see.
int64_t seen_keys(const AttendJob &j, const KvView &kv, int align);
// Scores kept per key and key head: a multiple of 4.
int score_rows(const AttendJob &j, const KvView &kv);
cudaError_t launch_attention_few(const AttendJob &j, const KvView &kv, cudaStream_t s);
// What joins their parts, once those are there.
cudaError_t launch_attention_few_finish(const AttendJob &j, const KvView &kv, cudaStream_t s);
// Of the others; whether that took a kernel that joins parts.
cudaError_t launch_attention_chunk(const AttendJob &j, const KvView &kv, cudaStream_t s, bool &joined);
// Their keys' mass, from lse2.
cudaError_t launch_attention_mass(const AttendJob &j, const KvView &kv, cudaStream_t s);

struct EvictJob {
    int budget, recent;
    const int32_t *new_table;
    int64_t new_stride;
    int32_t *new_lens;
};
cudaError_t launch_evict(const EvictJob &j, const KvView &kv, cudaStream_t s);

}  // namespace pv
