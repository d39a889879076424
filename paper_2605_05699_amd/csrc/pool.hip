// pool.hip -- the paged cache of one layer: its handle, the append (list of filled pages, window copies, quantizer) and the copies of
// pages and windows.  Attention over the pages is in pool_attention.hip.
#include <algorithm>
#include <memory>

#include "device_util.h"
#include "pool.h"

namespace {

// In front of the quantizer: workgroup 0 writes the list of the pages that the call fills, the others copy the tokens that stay in
// windows.  A window that is read for a filled page is never the one that tokens are copied into (the caller's two windows), so the
// two kernels need no order between their parts.  The list is in no fixed order (a counter in LDS); every page is quantized by itself, so the
// results do not depend on it.
constexpr int kWindowUnits = 1024;                           // of 16 bytes: what a workgroup copies at a time
__global__ void __launch_bounds__(256) srft_pool_window_kernel(const pool_append_args a, int U, int split, int most) {
    const pool_seqs& s = a.s;
    const int R = 1 << s.log_R;
    if (blockIdx.x == 0) {
        __shared__ int prefix[kPoolMaxSeqs + 1];
        __shared__ int wave_sums[4];
        __shared__ int listed;
        int base = 0;
        if (threadIdx.x == 0) listed = 0;
        // Exclusive sums of the candidates per sequence.  They stop at `most`, the entries that the workspace holds: starts that overlap count
        // new tokens more than once.
        for (int b0 = 0; b0 < s.n_seq; b0 += 256) {
            const int b = b0 + threadIdx.x;
            int n = 0;
            if (b < s.n_seq) {
                const pool_seq q = pool_seq_of(s, b);
                n = min(max((q.length >> s.log_R) - (max(q.before, 0) >> s.log_R), 0), most);
            }
            int sum = n;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int other = __shfl_up(sum, d);
                if ((int)(threadIdx.x & 63) >= d) sum = min(sum + other, most);
            }
            const int left = __shfl_up(sum, 1);
            if ((threadIdx.x & 63) == 63) wave_sums[threadIdx.x >> 6] = sum;
            __syncthreads();
            int before = base + ((threadIdx.x & 63) > 0 ? left : 0);
            for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before += wave_sums[w];
            base = min(base + wave_sums[0] + wave_sums[1] + wave_sums[2] + wave_sums[3], most);
            if (b < s.n_seq) prefix[b] = min(before, most);
            __syncthreads();
        }
        if (threadIdx.x == 0) prefix[s.n_seq] = base;
        __syncthreads();
        for (int f = threadIdx.x; f < base; f += 256) {
            int b = 0, end = s.n_seq;                        // the last sequence whose sum is not above f
            while (end - b > 1) {
                const int mid = (b + end) >> 1;
                if (prefix[mid] <= f) b = mid;
                else end = mid;
            }
            const pool_seq q = pool_seq_of(s, b);
            const int j = (max(q.before, 0) >> s.log_R) + f - prefix[b], held = max(q.before - j * R, 0);
            if (j >= s.max_pages) continue;
            const int page = s.table[b * s.max_pages + j], window = s.windows[2 * b];
            if (!pool_there(page, s.n_pages) || (held > 0 && !pool_there(window, s.n_windows))) continue;
            const int at = atomicAdd(&listed, 1);
            reinterpret_cast<i32x4*>(a.list + 4)[at] = i32x4{q.start + j * R - q.before, held, window, page};
        }
        __syncthreads();
        if (threadIdx.x == 0) a.list[0] = listed;
        return;
    }
    const int i = (blockIdx.x - 1) / split, part = (blockIdx.x - 1) % split, b = i >> 1;
    const bool v = i & 1;
    const pool_seq q = pool_seq_of(s, b);
    const int window = s.windows[2 * b + 1], first = max(max(q.full, q.before), 0), n = q.length - first;
    if (n <= 0 || !pool_there(window, s.n_windows)) return;
    const char* const from = v ? a.v : a.k;
    const long long token = v ? a.v_token : a.k_token, head = v ? a.v_head : a.k_head;
    uint4* const to = (uint4*)(v ? a.vb.window_f16_dev : a.kb.window_f16_dev) + (long long)window * a.heads * R * U;
    const int all = n * a.heads * U;
    for (int u0 = part * kWindowUnits + threadIdx.x; u0 < all; u0 += split * kWindowUnits) {
        uint4 x[kWindowUnits / 256];
        uint4* at[kWindowUnits / 256];
#pragma unroll
        for (int k = 0; k < kWindowUnits / 256; ++k) {       // (past the end the last unit again)
            const int u = min(u0 + 256 * k, all - 1), row = u / U, c = u - row * U, j = row / a.heads, h = row - j * a.heads;
            x[k] = reinterpret_cast<const uint4*>(from + (q.start + first - q.before + j) * token + h * head)[c];
            at[k] = to + ((h * R + first - q.full + j) * U + c);
        }
#pragma unroll
        for (int k = 0; k < kWindowUnits / 256; ++k) *at[k] = x[k];
    }
}

// Copies of pages and windows, in one launch: one workgroup per pair, pool and 32 KB, whose units are all on their way before the first is
// stored.  Bound by memory.  1500 pages of 20 KB in 16 layers: 185 us, 5.3 TB/s of reads and writes; with 16 KB a workgroup 208, with
// ordinary loads and stores, which leave in the L2 what nobody reads next, 194.
constexpr int kCopyPools = 64;
constexpr int kCopyUnits = 2048;                           // of 16 bytes, a workgroup's
constexpr int kCopyPairs = 1 << 22;                         // of pages and of windows in a launch, whose first dimension is limited to 2^32 threads
struct pool_copy_args {
    struct { char *codes, *scales, *window; } of[kCopyPools][2];
    struct { const int32_t* pairs; int n_pairs, count, units[2]; } what[2];  // pages, windows: numbers that exist; 16-byte units of codes and scales, or of a window and 0
};
static_assert(sizeof(pool_copy_args) <= 4096, "kernel arguments are limited to 4 KiB");
__global__ void __launch_bounds__(256) srft_pool_copy_kernel(const pool_copy_args a) {
    const bool windows = (int)blockIdx.x >= a.what[0].n_pairs;               // uniform
    const auto& w = a.what[windows];
    const long long pair = (int)blockIdx.x - (windows ? a.what[0].n_pairs : 0);
    const int from = w.pairs[2 * pair], to = w.pairs[2 * pair + 1];
    if (!pool_there(from, w.count) || !pool_there(to, w.count) || from == to) return;
    const auto& p = a.of[blockIdx.y];
    const int n = w.units[0] + w.units[1], all = 2 * n;
    const int u0 = (int)blockIdx.z * kCopyUnits + (int)threadIdx.x;
    if (u0 - (int)threadIdx.x >= all) return;                // (uniform: pages or windows, what is smaller)
    u32x4 x[kCopyUnits / 256];
    u32x4* at[kCopyUnits / 256];
#pragma unroll
    for (int i = 0; i < kCopyUnits / 256; ++i) {
        const int u = min(u0 + i * 256, all - 1), v = u >= n, k = u - v * n;
        const bool first = k < w.units[0];
        char* const base = windows ? p[v].window : first ? p[v].codes : p[v].scales;
        const int units = first ? w.units[0] : w.units[1], c = first ? k : k - w.units[0];
        x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base) + ((long long)from * units + c));
        at[i] = reinterpret_cast<u32x4*>(base) + ((long long)to * units + c);
    }
#pragma unroll
    for (int i = 0; i < kCopyUnits / 256; ++i)               // (what is past the end stores the last unit again)
        __builtin_nontemporal_store(x[i], at[i]);
}

bool known_page(int tokens) { return tokens >= 16 && tokens <= 256 && (tokens & (tokens - 1)) == 0; }

}  // namespace

int srft_pool_check(const srft_pool* p, const srft_paged_seqs* s, int64_t n_new) {
    if (!p || !s) return SRFT_ERR_NULL;
    if (s->n_seq < 0 || s->n_seq > kPoolMaxSeqs || s->max_new < 0 || s->max_length < 0 || s->max_length >= kPoolMaxLength || s->max_pages < 0 ||
        s->max_pages >= (1LL << 31) || s->max_pages < s->max_length / p->R || n_new < 0 || n_new * p->heads >= (1LL << 31))
        return SRFT_ERR_BAD_N;
    return SRFT_OK;
}
int srft_pool_check_pointers(const srft_paged_seqs* s) {
    if ((!s->page_table_dev && s->max_pages > 0) || !s->windows_dev || !s->lengths_dev || !s->starts_dev) return SRFT_ERR_NULL;
    for (const int32_t* p : {s->page_table_dev, s->windows_dev, s->lengths_dev, s->starts_dev})
        if (!srft_aligned(p, 4)) return SRFT_ERR_ALIGN;
    return SRFT_OK;
}

extern "C" {

int srft_pool_create(srft_pool_t** out, const srft_plan_t* plan_k, const srft_plan_t* plan_v, int n_heads, int page_tokens, int64_t n_pages,
                     int64_t n_windows, const srft_pool_buffers* k, const srft_pool_buffers* v) {
    if (!out) return SRFT_ERR_NULL;
    *out = nullptr;
    if (!plan_k || !plan_v || !k || !v) return SRFT_ERR_NULL;
    if (n_heads < 1 || n_heads > 1024 || !known_page(page_tokens) || n_heads * page_tokens % kTileVecs != 0 || n_pages < 0 || n_windows < 1 ||
        n_pages >= (1LL << 31) || n_windows >= (1LL << 31))
        return SRFT_ERR_BAD_N;
    if (!srft_plans_compatible(plan_k, plan_v)) return SRFT_ERR_MISMATCH;
    for (const srft_pool_buffers* b : {k, v}) {
        if (n_pages == 0 && (b->codes_dev || b->scales_dev)) return SRFT_ERR_BAD_N;
        if ((n_pages > 0 && (!b->codes_dev || !b->scales_dev)) || !b->window_f16_dev) return SRFT_ERR_NULL;
        if (!srft_aligned(b->codes_dev, 16) || !srft_aligned(b->scales_dev, 16) || !srft_aligned(b->window_f16_dev, 16)) return SRFT_ERR_ALIGN;
    }
    return srft_no_throw([&] {
        std::unique_ptr<srft_pool, int (*)(srft_pool*)> p(new srft_pool(), srft_pool_destroy);
        p->plan_k = plan_k;
        p->plan_v = plan_v;
        p->k = *k;
        p->v = *v;
        p->heads = n_heads;
        p->R = page_tokens;
        while ((1 << p->log_R) < page_tokens) ++p->log_R;
        p->n_pages = (int)n_pages;
        p->n_windows = (int)n_windows;
        const int rc = srft_pool_tables(p.get());
        if (rc == SRFT_OK) *out = p.release();
        return rc;
    });
}

int srft_pool_destroy(srft_pool_t* pool) {
    if (!pool) return SRFT_OK;
    const hipError_t e = pool->tables ? hipFree(pool->tables) : hipSuccess;
    delete pool;
    return e == hipSuccess ? (int)SRFT_OK : srft_hip_fail(e);
}

int64_t srft_pool_append_workspace_bytes(const srft_pool_t* pool, const srft_paged_seqs* seqs, int64_t n_new) {
    const int rc = srft_pool_check(pool, seqs, n_new);
    return rc != SRFT_OK ? rc : 16 + 16 * pool_fills(pool, seqs->n_seq, n_new);
}

int srft_pool_append(const srft_pool_t* pool, const srft_paged_seqs* seqs, const void* k_f16_dev, const void* v_f16_dev, int64_t n_new,
                     int64_t k_token, int64_t k_head, int64_t v_token, int64_t v_head, void* workspace_dev, void* hip_stream) {
    int rc = srft_pool_check(pool, seqs, n_new);
    if (rc != SRFT_OK) return rc;
    if (k_token % 8 || k_head % 8 || v_token % 8 || v_head % 8) return SRFT_ERR_ALIGN;
    const int64_t fills = pool_fills(pool, seqs->n_seq, n_new), page_tiles = (int64_t)pool->heads * pool->R / kTileVecs;
    if (fills * page_tiles * page_tiles >= (1LL << 31) || fills * pool->heads * pool->R >= (1LL << 31)) return SRFT_ERR_BAD_N;
    if (n_new == 0 || seqs->n_seq == 0) return SRFT_OK;
    rc = srft_pool_check_pointers(seqs);
    if (rc != SRFT_OK) return rc;
    if (!k_f16_dev || !v_f16_dev || !workspace_dev) return SRFT_ERR_NULL;
    if (!srft_aligned(k_f16_dev, 16) || !srft_aligned(v_f16_dev, 16) || !srft_aligned(workspace_dev, 16)) return SRFT_ERR_ALIGN;
    const srft_plan *pk = pool->plan_k, *pv = pool->plan_v;
    pool_append_args a;
    a.s = pool_seqs_of(pool, seqs, n_new);
    a.k = (const char*)k_f16_dev;
    a.v = (const char*)v_f16_dev;
    a.k_token = 2 * k_token, a.k_head = 2 * k_head, a.v_token = 2 * v_token, a.v_head = 2 * v_head;
    a.kb = pool->k;
    a.vb = pool->v;
    a.k_table = srft_plan_write_table(pk);
    a.v_table = srft_plan_write_table(pv);
    a.k_unscale = pk->unscale_w;
    a.v_unscale = pv->unscale_w;
    a.heads = pool->heads;
    a.gw = pk->gw;
    a.tiles_magic = srft_even_magic((int)page_tiles);
    a.list = (int*)workspace_dev;
    const hipStream_t st = (hipStream_t)hip_stream;
    // a workgroup for 16 KB of a window's new tokens, up to 4096 in all (with one for 32 tokens of it, 6 windows of up to 64 tokens at
    // d = 256 took 9.7 us, now 4.1)
    const int64_t units = (int64_t)std::min<int64_t>(seqs->max_new, pool->R) * pool->heads * pool->units();
    const int split = (int)std::max<int64_t>(1, std::min<int64_t>((units + kWindowUnits - 1) / kWindowUnits, 4096 / (2 * seqs->n_seq)));
    rc = srft_launch(srft_pool_window_kernel, dim3((unsigned)(1 + 2 * seqs->n_seq * split)), 256, st, a, pool->units(), split, (int)fills);
    if (rc != SRFT_OK) return rc;
    int threads = 0;
    const pool_append_kernel_t kernel = srft_plan_pool_append_kernel(pk, &threads);
    if (!kernel) return SRFT_ERR_BAD_D;
    const int64_t budget = std::clamp((pk->max_wgs > 0 ? pk->max_wgs : pk->grid_q) / 2, 1, 1 << 20);
    return srft_launch(kernel, dim3((unsigned)(2 * std::min(fills * page_tiles, budget))), threads, st, a);
}

int srft_pool_copy(const srft_pool_t* const* pools, int n_pools, const int32_t* pages_dev, int64_t n_page_pairs, const int32_t* windows_dev,
                   int64_t n_window_pairs, void* hip_stream) {
    const int64_t pairs = n_page_pairs + n_window_pairs;
    if (n_pools < 0 || n_page_pairs < 0 || n_window_pairs < 0 || n_page_pairs >= (1LL << 31) || n_window_pairs >= (1LL << 31) || pairs >= (1LL << 31))
        return SRFT_ERR_BAD_N;
    if (n_pools == 0) return SRFT_OK;
    if (!pools) return SRFT_ERR_NULL;
    for (int i = 0; i < n_pools; ++i) {
        if (!pools[i]) return SRFT_ERR_NULL;
        if (!srft_plans_compatible(pools[i]->plan_k, pools[0]->plan_k) || pools[i]->heads != pools[0]->heads || pools[i]->R != pools[0]->R ||
            pools[i]->n_pages != pools[0]->n_pages || pools[i]->n_windows != pools[0]->n_windows)
            return SRFT_ERR_MISMATCH;
    }
    if ((n_page_pairs > 0 && !pages_dev) || (n_window_pairs > 0 && !windows_dev)) return SRFT_ERR_NULL;
    if (!srft_aligned(pages_dev, 4) || !srft_aligned(windows_dev, 4)) return SRFT_ERR_ALIGN;
    if (pairs == 0) return SRFT_OK;
    const srft_pool* p = pools[0];
    const int rows = p->heads * p->R, d = p->plan_k->d;
    const auto some = [](int64_t all, int64_t from) { return (int)std::clamp<int64_t>(all - from, 0, kCopyPairs); };
    for (int64_t at = 0; at < std::max(n_page_pairs, n_window_pairs); at += kCopyPairs) {
        const int pages = some(n_page_pairs, at), windows = some(n_window_pairs, at);
        pool_copy_args a;
        a.what[0] = {pages_dev + 2 * at, pages, p->n_pages, {rows * d * p->plan_k->bits / 128, rows * (d / p->plan_k->g) / 4}};
        a.what[1] = {windows_dev + 2 * at, windows, p->n_windows, {rows * d / 8, 0}};
        const int units = 2 * std::max(pages ? a.what[0].units[0] + a.what[0].units[1] : 0, windows ? a.what[1].units[0] : 0);
        for (int i0 = 0; i0 < n_pools; i0 += kCopyPools) {
            const int n = std::min(kCopyPools, n_pools - i0);
            for (int i = 0; i < n; ++i)
                for (int v = 0; v < 2; ++v) {
                    const srft_pool_buffers& b = v ? pools[i0 + i]->v : pools[i0 + i]->k;
                    a.of[i][v] = {(char*)b.codes_dev, (char*)b.scales_dev, (char*)b.window_f16_dev};
                }
            const int rc = srft_launch(srft_pool_copy_kernel, dim3((unsigned)(pages + windows), (unsigned)n, (unsigned)((units + kCopyUnits - 1) / kCopyUnits)), 256, (hipStream_t)hip_stream, a);
            if (rc != SRFT_OK) return rc;
        }
    }
    return SRFT_OK;
}

}  // extern "C"
