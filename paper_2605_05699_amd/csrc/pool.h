// pool.h -- the paged cache of one layer: what its kernels and its host side share (pool.hip, kernels/pool_*.hip).
#ifndef SRFT_POOL_H
#define SRFT_POOL_H
#include "common.h"

constexpr int kPoolMaxSeqs = 4096;
constexpr int64_t kPoolMaxLength = 1LL << 30;

struct srft_pool {
    const srft_plan *plan_k = nullptr, *plan_v = nullptr;
    srft_pool_buffers k = {}, v = {};
    int heads = 0, R = 0, log_R = 0;
    int n_pages = 0, n_windows = 0;
    int decode_blocks[3][2] = {};           // workgroups of pool_decode that a compute unit holds: by form, for one and two blocks of rows
    uint4* tables = nullptr;                // device: the matrices of the queries and of the outputs (pool_attention.hip)
    float q_unscale = 1.0f, out_unscale = 1.0f;     // 2^-e of their scaling
    int units() const { return plan_k->d / 8; }             // 16-byte units of an fp16 row
};

// The sequences of a call as its kernels see them.  What the device arrays hold is cut to what the host has said, so that no
// value in them leads a kernel outside the buffers.
struct pool_seqs {
    const int32_t *table, *windows, *lengths, *starts;
    long long max_pages;
    int n_seq, max_new, max_length, n_new;
    int log_R, n_pages, n_windows;
};
struct pool_seq {
    int start, n_new, length, before, full;                  // rows of the new tokens; tokens with and without them; tokens in full pages
};
__device__ __forceinline__ pool_seq pool_seq_from(const pool_seqs& s, int start, int next_start, int length) {
    pool_seq q;
    q.start = min(max(start, 0), s.n_new);
    q.n_new = min(min(max(next_start, q.start), s.n_new) - q.start, s.max_new);
    q.length = min(max(length, 0), s.max_length);
    q.before = q.length - q.n_new;                           // (negative where there are more new tokens than tokens: those have no place)
    q.full = q.length >> s.log_R << s.log_R;
    return q;
}
__device__ __forceinline__ pool_seq pool_seq_of(const pool_seqs& s, int b) { return pool_seq_from(s, s.starts[b], s.starts[b + 1], s.lengths[b]); }
__device__ __forceinline__ bool pool_there(int number, int count) { return (unsigned)number < (unsigned)count; }

inline pool_seqs pool_seqs_of(const srft_pool* p, const srft_paged_seqs* s, int64_t n_new) {
    return {s->page_table_dev, s->windows_dev, s->lengths_dev, s->starts_dev, s->max_pages, s->n_seq, s->max_new, (int)s->max_length, (int)n_new,
            p->log_R, p->n_pages, p->n_windows};
}

// ---- append (kernels/pool_append_*.hip, pool.hip)
// Most pages that a call can fill, and its workspace: the number of filled pages, then an entry for each (srft_rows_pool).
inline int64_t pool_fills(const srft_pool* p, int n_seq, int64_t n_new) { return n_new / p->R + std::min<int64_t>(n_seq, n_new); }
struct pool_append_args {
    pool_seqs s;
    const char *k, *v;                                       // new tokens; strides in bytes
    long long k_token, k_head, v_token, v_head;
    srft_pool_buffers kb, vb;
    const uint4 *k_table, *v_table;
    float k_unscale, v_unscale;
    int heads, gw;
    uint32_t tiles_magic;
    int* list;                                               // workspace
};
typedef void (*pool_append_kernel_t)(const pool_append_args);
pool_append_kernel_t srft_pick_pool_append_plain(int d, int bits, int gm);
pool_append_kernel_t srft_pick_pool_append_fold(int d, int bits, int gm, bool fold4_q);

// the append's kernel for a plan's form of the write path
inline pool_append_kernel_t srft_plan_pool_append_kernel(const srft_plan* p, int* threads) {
    *threads = p->fold_q || p->fold4_q ? p->d : 2 * p->d / p->slabs_q;
    return p->fold_q || p->fold4_q ? srft_pick_pool_append_fold(p->d, p->bits, p->gm, p->fold4_q) : srft_pick_pool_append_plain(p->d, p->bits, p->gm);
}
// checks of the sequences of a call: their sizes, and their pointers
int srft_pool_check(const srft_pool* p, const srft_paged_seqs* s, int64_t n_new);
int srft_pool_check_pointers(const srft_paged_seqs* s);
// the device tables of attention (pool_attention.hip)
int srft_pool_tables(srft_pool* p);

#endif  // SRFT_POOL_H
