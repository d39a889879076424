// pool_attention.hip -- attention over a pool: its device tables, its workspace and its launches.
#include <algorithm>
#include <cmath>

#include "pool_attention.h"

namespace {

// Where each part of the workspace begins, and the grids that parts of it are counted by.
struct workspace {
    int64_t decode_before, chunk_before, blocks_before, q_rows, q_rows_low, q_factor, tail_rows, tail_factor, tail_columns, decode_parts, chunk_parts, bytes;
    int decode_grid, chunk_grid;
};
// Workgroups of a launch.  A cap on them (srft_plan_set_max_workgroups) may change between the call that sizes a workspace and the one that
// uses it: it makes launches smaller, never larger, and the workspace is for launches without one.
int workgroups(const srft_pool* p, int per_unit) {
    const int all = p->plan_k->compute_units * per_unit;
    return p->plan_k->max_wgs > 0 ? std::min(p->plan_k->max_wgs, all) : all;
}
constexpr int kChunkRows = kPoolBlock * kPoolChunkWaves;
// blocks of kChunkRows rows of all sequences, at most, where those with fewer than `least` rows count for none
int64_t row_blocks(const srft_paged_seqs* s, int64_t n_new, int group, int least) {
    const int64_t rows = n_new * group;
    return rows / kChunkRows + std::min<int64_t>(s->n_seq, rows / least);
}
// Sequences that bring few rows a key head go to pool_decode, cb blocks of 16 of them a workgroup, the others to pool_chunk.  Two blocks where
// a sequence may bring 17 to 32 rows and none brings more, up to d = 128 (beyond it two blocks' sums do not fit the registers: there a
// workgroup takes one block, and the keys are read twice); else one, and 17 rows are a chunk.
struct split {
    int cb, rows;
    bool chunk, decode;
};
split split_of(const srft_paged_seqs* s, int64_t n_new, int group, int d) {
    const int64_t most = std::min<int64_t>(s->max_new, n_new) * group;
    const bool few = most > 16 && most <= kPoolDecodeRows;
    const int rows = few ? kPoolDecodeRows : 16;
    return {few && d <= 128 ? 2 : 1, rows, most > rows, most <= rows || s->n_seq > 1 || n_new * group <= rows};
}
workspace layout(const srft_pool* p, const srft_paged_seqs* s, int64_t n_new, int q_heads) {
    const int d = p->plan_k->d, group = q_heads / p->heads;
    const int64_t tail = 2LL * s->n_seq * p->heads * p->R, rows = n_new * q_heads;
    workspace w;
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const split s16 = split_of(s, n_new, group, d);
    const int cus = p->plan_k->compute_units, per_unit = p->decode_blocks[s16.cb - 1];
    w.decode_grid = workgroups(p, per_unit);
    w.chunk_grid = workgroups(p, 1);
    w.decode_before = take(4LL * (s->n_seq + 1));
    w.chunk_before = take(4LL * (s->n_seq + 1));
    w.blocks_before = take(4LL * (s->n_seq + 1));
    w.q_rows = take(2 * rows * d);
    w.q_rows_low = take(2 * rows * d);
    w.q_factor = take(4 * rows);
    w.tail_rows = take(2 * tail * d);
    w.tail_factor = take(4 * tail);
    w.tail_columns = take(tail * d);
    w.decode_parts = take(2LL * cus * per_unit * s16.cb * (16 * d + 3 * 64) * 4);
    w.chunk_parts = take(s16.chunk ? 2LL * cus * kPoolChunkWaves * pool_part(d) * 4 : 0);
    w.bytes = at;
    return w;
}

pool_attention_kernel_t srft_pool_decode_kernel_of(const srft_plan* p, int cb) {
    return p->bits == 8 ? srft_pick_pool_decode_b8(p->d, cb, p->gm) : srft_pick_pool_decode_b4(p->d, cb, p->gm);
}

int check(const srft_pool* pool, const srft_paged_seqs* seqs, int64_t n_new, int q_heads) {
    const int rc = srft_pool_check(pool, seqs, n_new);
    if (rc != SRFT_OK) return rc;
    if (q_heads < 1 || q_heads % pool->heads != 0 || q_heads > 64 * pool->heads || n_new * q_heads >= (1LL << 31) - 32) return SRFT_ERR_BAD_N;
    // units of work (kPoolMostUnits), tiles and workgroups are counted with 32 bits
    const int d = pool->plan_k->d, group = q_heads / pool->heads;
    const int64_t most = kPoolMostUnits, tiles = seqs->max_length / 32 + 2, heads = (int64_t)seqs->n_seq * pool->heads;
    const int64_t blocks = n_new * group / kChunkRows + seqs->n_seq;
    if (2 * heads * tiles >= most || blocks * pool->heads * std::max<int64_t>(tiles, kPoolChunkWaves) >= most ||
        (heads * pool->R / kTileVecs * 2 + pool->plan_k->compute_units * 3 + 1) * 2 * d > UINT32_MAX)        // (threads of pool_rotate)
        return SRFT_ERR_BAD_N;
    return SRFT_OK;
}

}  // namespace

// Both tables are R_k^T and R_v as fp16 hi + lo fragments.  The queries': [D / 32 slabs][D / 16 k-steps][hi, lo][64 lanes], as on the
// write path (lane l: row slab_output_of_row(l % 32), columns 16 t + 8 (l / 32) + e).  The outputs': the same with the columns
// in the order that sums of values have them in a lane, 16 t + 8 (e / 4) + 4 (l / 32) + e % 4, positions instead of channels.  The
// outputs' again for blocks of 16 rows, [D / 16][D / 32 k-steps][hi, lo][64 lanes]: row l % 16, channels 32 t + 16 (e / 4) + 4 (l / 16) + e % 4.
int srft_pool_tables(srft_pool* p) {
    const int d = p->plan_k->d, G = d / 32, T = d / 16, bits = p->plan_k->bits;
    std::vector<float> rk((size_t)d * d), rv((size_t)d * d);                // [channel][n]
    int device = 0;
    SRFT_HIP(hipGetDevice(&device));
    if (device != p->plan_k->device) return SRFT_ERR_MISMATCH;
    SRFT_HIP(hipMemcpy(rk.data(), p->plan_k->rmat_f32, rk.size() * 4, hipMemcpyDeviceToHost));
    SRFT_HIP(hipMemcpy(rv.data(), p->plan_v->rmat_f32, rv.size() * 4, hipMemcpyDeviceToHost));
    std::vector<double> q((size_t)d * d), o((size_t)d * d);
    for (int k = 0; k < d; ++k)
        for (int n = 0; n < d; ++n) {
            q[(size_t)k * d + n] = rk[(size_t)k * d + n];
            o[(size_t)n * d + k] = rv[(size_t)k * d + n];
        }
    std::vector<uint16_t> qh, ql, oh, ol;
    p->q_unscale = (float)std::ldexp(1.0, -srft_split_hi_lo(q, qh, ql));
    p->out_unscale = (float)std::ldexp(1.0, -srft_split_hi_lo(o, oh, ol));
    const size_t units = (size_t)G * T * 2 * 64;
    std::vector<uint16_t> image(3 * units * 8);
    static const int byte_order[8] = {0, 2, 1, 3, 4, 6, 5, 7};
    for (int w = 0; w < G; ++w)
        for (int t = 0; t < T; ++t)
            for (int l = 0; l < 64; ++l)
                for (int e = 0; e < 8; ++e) {
                    const int row = 32 * w + srft_slab_output_of_row(l % 32), h = l / 32;
                    const size_t at = (((size_t)w * T + t) * 2 * 64 + l) * 8 + e, src = (size_t)row * d + 16 * t + 8 * h + e;
                    image[at] = qh[src];
                    image[at + 64 * 8] = ql[src];
                    const int in8 = 4 * h + e % 4, channel = 16 * t + 8 * (e / 4) + (bits == 8 ? byte_order[in8] : in8 / 2 + 4 * (in8 % 2));
                    image[units * 8 + at] = oh[(size_t)row * d + channel];
                    image[units * 8 + at + 64 * 8] = ol[(size_t)row * d + channel];
                }
    for (int n = 0; n < d / 16; ++n)
        for (int t = 0; t < G; ++t)
            for (int l = 0; l < 64; ++l)
                for (int e = 0; e < 8; ++e) {
                    const size_t at = 2 * units * 8 + (((size_t)n * G + t) * 2 * 64 + l) * 8 + e;
                    const size_t src = (size_t)(16 * n + l % 16) * d + 32 * t + 16 * (e / 4) + 4 * (l / 16) + e % 4;
                    image[at] = oh[src];
                    image[at + 64 * 8] = ol[src];
                }
    // The scans read page 0 in the place of one that does not exist (and count it for nothing): where there is none, zeros behind the tables.
    const size_t rows = p->n_pages > 0 ? 0 : (size_t)p->heads * p->R, code_bytes = rows * d * bits / 8, scale_bytes = rows * (d / p->plan_k->g) * 4;
    const size_t table_bytes = image.size() * 2;
    image.resize((table_bytes + code_bytes + scale_bytes) / 2);
    for (int cb = 1; cb <= 2; ++cb) {
        SRFT_HIP(hipOccupancyMaxActiveBlocksPerMultiprocessor(&p->decode_blocks[cb - 1], (const void*)srft_pool_decode_kernel_of(p->plan_k, cb), 64 * kPoolTeam, 0));
        p->decode_blocks[cb - 1] = std::max(1, std::min(4, p->decode_blocks[cb - 1]));
    }
    SRFT_HIP(hipMalloc((void**)&p->tables, image.size() * 2));
    SRFT_HIP(hipMemcpy(p->tables, image.data(), image.size() * 2, hipMemcpyHostToDevice));
    if (rows > 0)
        for (srft_pool_buffers* b : {&p->k, &p->v}) {
            b->codes_dev = (uint8_t*)p->tables + table_bytes;
            b->scales_dev = (float*)(b->codes_dev + code_bytes);
        }
    return SRFT_OK;
}

extern "C" {

int64_t srft_pool_attention_workspace_bytes(const srft_pool_t* pool, const srft_paged_seqs* seqs, int64_t n_new, int n_q_heads) {
    const int rc = check(pool, seqs, n_new, n_q_heads);
    return rc != SRFT_OK ? rc : layout(pool, seqs, n_new, n_q_heads).bytes;
}

int srft_pool_attention(const srft_pool_t* pool, const srft_paged_seqs* seqs, const void* q_dev, int type, int64_t n_new, int n_q_heads,
                        int64_t q_token, int64_t q_head, float softmax_scale, void* out_dev, int64_t out_token, int64_t out_head,
                        void* workspace_dev, void* hip_stream) {
    int rc = check(pool, seqs, n_new, n_q_heads);
    if (rc != SRFT_OK) return rc;
    if ((type != SRFT_F16 && type != SRFT_BF16) || !std::isfinite(softmax_scale)) return SRFT_ERR_BAD_N;
    if (q_token % 8 || q_head % 8 || out_token % 8 || out_head % 8) return SRFT_ERR_ALIGN;
    if (n_new == 0 || seqs->n_seq == 0) return SRFT_OK;
    rc = srft_pool_check_pointers(seqs);
    if (rc != SRFT_OK) return rc;
    if (!q_dev || !out_dev || !workspace_dev) return SRFT_ERR_NULL;
    if (!srft_aligned(q_dev, 16) || !srft_aligned(out_dev, 16) || !srft_aligned(workspace_dev, 256)) return SRFT_ERR_ALIGN;
    const srft_plan *pk = pool->plan_k, *pv = pool->plan_v;
    const int d = pk->d, group = n_q_heads / pool->heads;
    const workspace w = layout(pool, seqs, n_new, n_q_heads);
    const split sp = split_of(seqs, n_new, group, d);
    char* const base = (char*)workspace_dev;
    pool_attention_args a;
    a.s = pool_seqs_of(pool, seqs, n_new);
    a.kb = pool->k;
    a.vb = pool->v;
    a.heads = pool->heads;
    a.group = group;
    a.g = pk->g;
    a.q = (const char*)q_dev;
    a.out = (char*)out_dev;
    a.q_token = 2 * q_token, a.q_head = 2 * q_head, a.out_token = 2 * out_token, a.out_head = 2 * out_head;
    a.bf16 = type == SRFT_BF16;
    a.exponent = std::fabs(softmax_scale) * 1.44269504088896340736f;
    a.sign = softmax_scale < 0 ? -1.0f : 1.0f;
    a.q_table = pool->tables;
    const size_t units = (size_t)(d / 32) * (d / 16) * 2 * 64;
    a.out_table = pool->tables + units;
    a.out_table16 = pool->tables + 2 * units;
    a.k_table = pk->wfrag;
    a.v_table = pv->wfrag;
    a.q_unscale = pool->q_unscale;
    a.out_unscale = pool->out_unscale;
    a.k_unscale = pk->unscale_w;
    a.v_unscale = pv->unscale_w;
    a.q_tiles = (int)((n_new * n_q_heads + kTileVecs - 1) / kTileVecs);
    // as many as a compute unit's registers hold at a time, each with the matrix for all its passes (65,536 rows of d = 128: 12.4 us, with two
    // a unit 13.0, with four 14.3; 32,000 of d = 256: 23.4, with two 26.2)
    a.q_grid = std::min(a.q_tiles, workgroups(pool, d <= 128 ? 3 : 1));
    a.decode_before = (int*)(base + w.decode_before);
    a.chunk_before = (int*)(base + w.chunk_before);
    a.blocks_before = sp.chunk ? (int*)(base + w.blocks_before) : nullptr;
    a.q_rows = (unsigned short*)(base + w.q_rows);
    a.q_factor = (float*)(base + w.q_factor);
    a.tail_rows = (unsigned short*)(base + w.tail_rows);
    a.tail_factor = (float*)(base + w.tail_factor);
    a.tail_columns = (unsigned short*)(base + w.tail_columns);
    a.decode_parts = (float*)(base + w.decode_parts);
    a.chunk_parts = (float*)(base + w.chunk_parts);
    a.q_rows_low = sp.decode ? (unsigned short*)(base + w.q_rows_low) : nullptr;     // (chunks do not read them)
    a.decode_grid = w.decode_grid;
    a.decode_rows = sp.decode ? sp.rows : 0;                 // (0: the one sequence there is goes to pool_chunk, however few tokens it brings)
    a.decode_block = 16 * sp.cb;
    a.decode_keys = pool_decode_keys(d, sp.cb);
    a.chunk_grid = w.chunk_grid;
    const hipStream_t st = (hipStream_t)hip_stream;
    const int tail_tiles = 2 * seqs->n_seq * (pool->heads * pool->R / kTileVecs), heads = seqs->n_seq * pool->heads;
    rc = srft_launch(srft_pick_pool_rotate(d, pk->bits), dim3((unsigned)(1 + a.q_grid + tail_tiles)), 2 * d, st, a);
    if (rc == SRFT_OK && sp.chunk) rc = srft_launch(srft_pick_pool_chunk(d, pk->bits), dim3((unsigned)a.chunk_grid), 64 * kPoolChunkWaves, st, a);
    if (rc == SRFT_OK && sp.decode) rc = srft_launch(srft_pool_decode_kernel_of(pk, sp.cb), dim3((unsigned)a.decode_grid), 64 * kPoolTeam, st, a);
    a.decode_merges = sp.decode ? heads * ((a.decode_rows + a.decode_block - 1) / a.decode_block) : 0;
    a.merges = (unsigned)a.decode_merges + (sp.chunk ? (unsigned)(row_blocks(seqs, n_new, group, a.decode_rows + 1) * pool->heads * kPoolChunkWaves) : 0);
    if (rc == SRFT_OK && a.merges) rc = srft_launch(srft_pick_pool_merge(d, sp.cb), srft_grid(a.merges), 64 * kPoolTeam, st, a);
    return rc;
}

}  // extern "C"
