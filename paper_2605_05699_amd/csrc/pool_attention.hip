// pool_attention.hip -- attention over a pool: its device tables, its workspace and its launches.
#include <algorithm>
#include <cmath>

#include "pool_attention.h"

namespace {

// What a call is, beside the sequences.
struct form_of_call {
    int form = kPoolCausal;
    int64_t recent = kPoolMaxLength, sinks = 0;
    const srft_shared_prefixes* prefixes = nullptr;
    int groups() const { return form == kPoolShared ? prefixes->n_groups : 0; }
};

// Where each part of the workspace begins, and the grids that parts of it are counted by.
struct workspace {
    int64_t bounds, items, joint_rows[2], joint_heads[2];
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
// Sequences that bring few rows a key head go to pool_decode, cb blocks of 16 of them a workgroup, the others to pool_chunk.  Two blocks where
// a sequence may bring 17 to 32 rows and none brings more, up to d = 128 (beyond it two blocks' sums do not fit the registers: there a
// workgroup takes one block, and the keys are read twice); else one, and 17 rows are a chunk.
// A group's tokens in common go to pool_decode, in blocks that each read the keys, up to kCommonRows rows; and in calls of up to kFewRows rows, which
// need no launch for chunks then.  With up to 16 in place of kCommonRows six samples of 800 tokens take 40 us (now 22) and five prompts with 2 to 11
// samples at d = 256 96 (now 67); with up to 96 six groups of 96 rows behind 4000 tokens take 85 (now 78; d = 256 134, now 115), one alone 27 (as
// now; as a chunk 45) and behind 16,384 tokens 49 (56).  128 rows in one group: 30 us behind 2000 tokens (as a chunk 46), 58 (58) behind 16,384, at d
// = 256 52 (73) and 107 (100); 192: 31 (51), 72 (64), 54 (79), 133 (106).
constexpr int kCommonRows = 48, kFewRows = 128;
struct split {
    int cb, rows, common_rows;
    bool chunk, decode;
};
split split_of(const srft_paged_seqs* s, const form_of_call& f, int64_t n_new, int group, int d) {
    const int64_t most = std::min<int64_t>(s->max_new, n_new) * group;
    const bool few = most > 16 && most <= kPoolDecodeRows;
    const int rows = few ? kPoolDecodeRows : 16;
    // (a group's tokens in common have the rows of all its sequences)
    const int common = n_new * group <= kFewRows ? kFewRows : kCommonRows;
    return {few && d <= 128 ? 2 : 1, rows, common, most > rows || (f.groups() > 0 && n_new * group > common), most <= rows || s->n_seq > 1 || n_new * group <= rows};
}
workspace layout(const srft_pool* p, const srft_paged_seqs* s, const form_of_call& f, int64_t n_new, int q_heads) {
    const int d = p->plan_k->d, group = q_heads / p->heads, items = s->n_seq + f.groups();
    const int64_t tail = 2LL * s->n_seq * p->heads * p->R, rows = n_new * q_heads;
    workspace w = {};
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const split s16 = split_of(s, f, n_new, group, d);
    const int cus = p->plan_k->compute_units, per_unit = p->decode_blocks[f.form][s16.cb - 1];
    w.decode_grid = workgroups(p, per_unit);
    w.chunk_grid = workgroups(p, 1);
    w.decode_before = take(4LL * (items + 1));
    w.chunk_before = take(4LL * (items + 1));
    w.blocks_before = take(4LL * (items + 1));
    w.q_rows = take(2 * rows * d);
    w.q_rows_low = take(2 * rows * d);
    w.q_factor = take(4 * rows);
    w.tail_rows = take(2 * tail * d);
    w.tail_factor = take(4 * tail);
    w.tail_columns = take(tail * d);
    w.decode_parts = take(2LL * cus * per_unit * s16.cb * (16 * d + 3 * 64) * 4);
    w.chunk_parts = take(s16.chunk ? 2LL * cus * kPoolChunkWaves * pool_part(d) * 4 : 0);
    if (f.groups() > 0) {
        w.bounds = take(4LL * (f.groups() + 1));
        w.items = take((int64_t)sizeof(pool_item) * items);
        for (int i = 0; i < 2; ++i) {
            w.joint_rows[i] = take(4 * rows * d);
            w.joint_heads[i] = take(16 * rows);
        }
    }
    w.bytes = at;
    return w;
}

pool_attention_kernel_t srft_pool_decode_kernel_of(const srft_plan* p, int cb, int form) {
    if (form == kPoolSliding) return p->bits == 8 ? srft_pick_pool_decode_sliding_b8(p->d, cb, p->gm) : srft_pick_pool_decode_sliding_b4(p->d, cb, p->gm);
    if (form == kPoolShared) return p->bits == 8 ? srft_pick_pool_decode_shared_b8(p->d, cb, p->gm) : srft_pick_pool_decode_shared_b4(p->d, cb, p->gm);
    return p->bits == 8 ? srft_pick_pool_decode_b8(p->d, cb, p->gm) : srft_pick_pool_decode_b4(p->d, cb, p->gm);
}
pool_attention_kernel_t srft_pool_chunk_kernel_of(const srft_plan* p, int form) {
    return form == kPoolSliding ? srft_pick_pool_chunk_sliding(p->d, p->bits)
           : form == kPoolShared ? srft_pick_pool_chunk_shared(p->d, p->bits) : srft_pick_pool_chunk(p->d, p->bits);
}

int check(const srft_pool* pool, const srft_paged_seqs* seqs, const form_of_call& f, int64_t n_new) {
    if (f.form == kPoolShared && !f.prefixes) return SRFT_ERR_NULL;
    const int rc = srft_pool_check(pool, seqs, n_new);
    if (rc != SRFT_OK) return rc;
    return f.recent < 1 || f.sinks < 0 || f.groups() < 0 || f.groups() > seqs->n_seq || (f.prefixes && f.prefixes->reserved != 0) ? SRFT_ERR_BAD_N : SRFT_OK;
}
// The form that answers a call: what sees everything, and groups of none, are the causal form.
form_of_call answering(const srft_paged_seqs* s, const form_of_call& f) {
    const bool all = f.form == kPoolSliding && std::min(f.recent, kPoolMaxLength) + std::min(f.sinks, kPoolMaxLength) >= s->max_length;
    return all || (f.form == kPoolShared && f.groups() == 0) ? form_of_call{} : f;
}
int check_sizes(const srft_pool* pool, const srft_paged_seqs* seqs, const form_of_call& f, int64_t n_new, int q_heads) {
    if (q_heads < 1 || q_heads % pool->heads != 0 || q_heads > 64 * pool->heads || n_new * q_heads >= (1LL << 31) - 32) return SRFT_ERR_BAD_N;
    // units of work (kPoolMostUnits), tiles and workgroups are counted with 32 bits
    const int d = pool->plan_k->d, group = q_heads / pool->heads;
    const int64_t most = kPoolMostUnits, tiles = seqs->max_length / 32 + 2 + (f.form == kPoolCausal ? 0 : kPoolChunkStart<kPoolSliding>), heads = (int64_t)seqs->n_seq * pool->heads;
    const int64_t items = seqs->n_seq + f.groups(), blocks = (f.groups() > 0 ? 2 : 1) * n_new * group / kChunkRows + items;
    if ((f.groups() > 0 ? 3 * items + kFewRows / 16 : 2 * items) * pool->heads * tiles >= most || blocks * pool->heads * std::max<int64_t>(tiles, kPoolChunkWaves) >= most ||
        (heads * pool->R / kTileVecs * 2 + pool->plan_k->compute_units * 3 + 1) * 2 * d > UINT32_MAX)        // (threads of pool_rotate)
        return SRFT_ERR_BAD_N;
    return SRFT_OK;
}

int64_t bytes_of(const srft_pool* pool, const srft_paged_seqs* seqs, const form_of_call& f, int64_t n_new, int q_heads) {
    int rc = check(pool, seqs, f, n_new);
    if (rc != SRFT_OK) return rc;
    const form_of_call by = answering(seqs, f);
    rc = check_sizes(pool, seqs, by, n_new, q_heads);
    return rc != SRFT_OK ? rc : layout(pool, seqs, by, n_new, q_heads).bytes;
}

int attend(const srft_pool* pool, const srft_paged_seqs* seqs, form_of_call f, const void* q_dev, int type, int64_t n_new, int n_q_heads, int64_t q_token,
           int64_t q_head, float softmax_scale, void* out_dev, int64_t out_token, int64_t out_head, void* workspace_dev, void* hip_stream) {
    int rc = check(pool, seqs, f, n_new);
    if (rc != SRFT_OK) return rc;
    f = answering(seqs, f);
    rc = check_sizes(pool, seqs, f, n_new, n_q_heads);
    if (rc != SRFT_OK) return rc;
    if ((type != SRFT_F16 && type != SRFT_BF16) || !std::isfinite(softmax_scale)) return SRFT_ERR_BAD_N;
    if (q_token % 8 || q_head % 8 || out_token % 8 || out_head % 8) return SRFT_ERR_ALIGN;
    if (n_new == 0 || seqs->n_seq == 0) return SRFT_OK;
    rc = srft_pool_check_pointers(seqs);
    if (rc != SRFT_OK) return rc;
    if (f.groups() > 0) {
        if (!f.prefixes->groups_dev || !f.prefixes->tokens_dev) return SRFT_ERR_NULL;
        if (!srft_aligned(f.prefixes->groups_dev, 4) || !srft_aligned(f.prefixes->tokens_dev, 4)) return SRFT_ERR_ALIGN;
    }
    if (!q_dev || !out_dev || !workspace_dev) return SRFT_ERR_NULL;
    if (!srft_aligned(q_dev, 16) || !srft_aligned(out_dev, 16) || !srft_aligned(workspace_dev, 256)) return SRFT_ERR_ALIGN;
    const srft_plan *pk = pool->plan_k, *pv = pool->plan_v;
    const int d = pk->d, group = n_q_heads / pool->heads;
    const workspace w = layout(pool, seqs, f, n_new, n_q_heads);
    const split sp = split_of(seqs, f, n_new, group, d);
    char* const base = (char*)workspace_dev;
    pool_attention_args a = {};
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
    a.recent = (int)std::min(f.recent, kPoolMaxLength);
    a.sinks = (int)std::min(f.sinks, kPoolMaxLength);
    a.bits = pk->bits;
    if (f.groups() > 0) {
        a.groups = f.prefixes->groups_dev;
        a.shared = f.prefixes->tokens_dev;
        a.n_groups = f.groups();
        a.common_rows = sp.common_rows;
        a.bounds = (int*)(base + w.bounds);
        a.items = (pool_item*)(base + w.items);
        for (int i = 0; i < 2; ++i) {
            a.joint_rows[i] = (float*)(base + w.joint_rows[i]);
            a.joint_heads[i] = (float*)(base + w.joint_heads[i]);
        }
    }
    const hipStream_t st = (hipStream_t)hip_stream;
    const int tail_tiles = 2 * seqs->n_seq * (pool->heads * pool->R / kTileVecs);
    rc = srft_launch(srft_pick_pool_rotate(d, pk->bits, f.form), dim3((unsigned)(1 + a.q_grid + tail_tiles)), 2 * d, st, a);
    if (rc == SRFT_OK && sp.chunk) rc = srft_launch(srft_pool_chunk_kernel_of(pk, f.form), dim3((unsigned)a.chunk_grid), 64 * kPoolChunkWaves, st, a);
    if (rc == SRFT_OK && sp.decode) rc = srft_launch(srft_pool_decode_kernel_of(pk, sp.cb, f.form), dim3((unsigned)a.decode_grid), 64 * kPoolTeam, st, a);
    const int64_t rows = n_new * group;
    a.decode_merges = sp.decode ? seqs->n_seq * pool->heads * ((a.decode_rows + a.decode_block - 1) / a.decode_block) : 0;
    a.merges = (unsigned)a.decode_merges +
               (sp.chunk ? (unsigned)((rows / kChunkRows + std::min<int64_t>(seqs->n_seq, rows / (a.decode_rows + 1))) * pool->heads * kPoolChunkWaves) : 0);
    if (rc == SRFT_OK && a.merges) rc = srft_launch(srft_pick_pool_merge(d, sp.cb, f.form), srft_grid(a.merges), 64 * kPoolTeam, st, a);
    return rc;
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
    for (int form = 0; form < kPoolForms; ++form)
        for (int cb = 1; cb <= 2; ++cb) {
            int& blocks = p->decode_blocks[form][cb - 1];
            SRFT_HIP(hipOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, (const void*)srft_pool_decode_kernel_of(p->plan_k, cb, form), 64 * kPoolTeam, 0));
            blocks = std::max(1, std::min(4, blocks));
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
    return bytes_of(pool, seqs, {}, n_new, n_q_heads);
}
int srft_pool_attention(const srft_pool_t* pool, const srft_paged_seqs* seqs, const void* q_dev, int type, int64_t n_new, int n_q_heads,
                        int64_t q_token, int64_t q_head, float softmax_scale, void* out_dev, int64_t out_token, int64_t out_head,
                        void* workspace_dev, void* hip_stream) {
    return attend(pool, seqs, {}, q_dev, type, n_new, n_q_heads, q_token, q_head, softmax_scale, out_dev, out_token, out_head, workspace_dev, hip_stream);
}

int64_t srft_pool_attention_sliding_workspace_bytes(const srft_pool_t* pool, const srft_paged_seqs* seqs, int64_t n_new, int n_q_heads) {
    // (of the least reach, and of one that sees everything: that is the causal form, whose scan may have more workgroups)
    const int64_t all = bytes_of(pool, seqs, {}, n_new, n_q_heads), some = bytes_of(pool, seqs, {kPoolSliding, 1, 0}, n_new, n_q_heads);
    return std::min(all, some) < 0 ? std::min(all, some) : std::max(all, some);
}
int srft_pool_attention_sliding(const srft_pool_t* pool, const srft_paged_seqs* seqs, const void* q_dev, int type, int64_t n_new, int n_q_heads,
                                int64_t q_token, int64_t q_head, float softmax_scale, int64_t recent, int64_t sinks, void* out_dev,
                                int64_t out_token, int64_t out_head, void* workspace_dev, void* hip_stream) {
    return attend(pool, seqs, {kPoolSliding, recent, sinks}, q_dev, type, n_new, n_q_heads, q_token, q_head, softmax_scale, out_dev, out_token, out_head,
                  workspace_dev, hip_stream);
}

int64_t srft_pool_attention_shared_workspace_bytes(const srft_pool_t* pool, const srft_paged_seqs* seqs, const srft_shared_prefixes* prefixes,
                                                   int64_t n_new, int n_q_heads) {
    return bytes_of(pool, seqs, {kPoolShared, kPoolMaxLength, 0, prefixes}, n_new, n_q_heads);
}
int srft_pool_attention_shared(const srft_pool_t* pool, const srft_paged_seqs* seqs, const srft_shared_prefixes* prefixes, const void* q_dev, int type,
                               int64_t n_new, int n_q_heads, int64_t q_token, int64_t q_head, float softmax_scale, void* out_dev,
                               int64_t out_token, int64_t out_head, void* workspace_dev, void* hip_stream) {
    return attend(pool, seqs, {kPoolShared, kPoolMaxLength, 0, prefixes}, q_dev, type, n_new, n_q_heads, q_token, q_head, softmax_scale, out_dev, out_token,
                  out_head, workspace_dev, hip_stream);
}

}  // extern "C"
