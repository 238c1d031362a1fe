/* In the place of libpvmvmd.so for the binding's native module (csrc/calls.c): the
 * calls with a batch return its T, read once two of them are under way.  Driven by
 * test_calls_threads.py. */
#include <stdatomic.h>
#include <time.h>

#include "pvmvmd.h"

static atomic_int g_inside;

static int rows_seen(const pvmvmd_kv_batch *batch) {
    atomic_fetch_add(&g_inside, 1);
    for (int i = 0; i < 5000 && atomic_load(&g_inside) < 2; ++i)
        nanosleep(&(struct timespec){0, 1000000}, NULL);
    return atomic_load(&g_inside) < 2 ? -1 : batch->T;
}
void stub_reset(void) { atomic_store(&g_inside, 0); }

int pvmvmd_rope(const pvmvmd_rope_view *rope, const int32_t *pos_dev, int T, int H, int D, const void *x_dev,
                int x_type, int64_t x_token, int64_t x_head, float scale, void *out_dev, int out_type,
                int64_t out_token, int64_t out_head, void *stream) {
    return PVMVMD_OK;
}
int pvmvmd_kv_append(const pvmvmd_kv_pool *pool, const pvmvmd_kv_batch *batch, const pvmvmd_rope_view *rope,
                     const int32_t *pos_dev, int in_type, float scale, const void *k_dev, int64_t k_token,
                     int64_t k_head, const void *v_dev, int64_t v_token, int64_t v_head, int Hq, const void *q_dev,
                     int64_t q_token, int64_t q_head, void *q_out_dev, int64_t q_out_token, int64_t q_out_head,
                     void *stream) {
    return rows_seen(batch);
}
int pvmvmd_paged_attention(const pvmvmd_kv_pool *pool, const pvmvmd_kv_batch *batch, int Hq, const void *q_dev,
                           int64_t q_token, int64_t q_head, float scale, int causal, int window, int accumulate,
                           void *out_dev, int64_t out_token, int64_t out_head, float *lse_dev, void *stream) {
    return rows_seen(batch);
}
int pvmvmd_kv_evict(const pvmvmd_kv_pool *pool, const pvmvmd_kv_batch *batch, int budget, int recent,
                    const int32_t *new_table_dev, int64_t new_table_stride, int new_max_pages, int32_t *new_lens_dev,
                    void *stream) {
    return PVMVMD_OK;
}
