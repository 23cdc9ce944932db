// What the entry points for several sequences share: argument checks, and a batch as the kernels take it.
#pragma once
#include <algorithm>
#include <cmath>
#include <hip/hip_runtime.h>

#include "card.h"
#include "card_attend.hip"

namespace card {

inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
inline int launch_status() { return hipGetLastError() == hipSuccess ? CARD_OK : CARD_EDEVICE; }
inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
// Of a layer of a pool with 16 or 4 bits a value.
inline size_t layer_bytes(const card_model_cfg* cfg, int32_t n_pages, int bits) { return size_t(n_pages) * cfg->n_kv_heads * (bits == 16 ? 32 : 9) * cfg->head_dim; }

inline bool rows_ok(const card_rows* r, int32_t type, int64_t least_stride) {
    const int64_t unit = type == CARD_F32 ? 4 : 8;
    return r && r->data && r->type == type && aligned16(r->data) && r->row_stride >= least_stride && r->head_stride >= least_stride &&
           r->row_stride % unit == 0 && r->head_stride % unit == 0;
}

// A launch has less than 2^32 threads in x: 2^24 workgroups of 256.  (units of 16 rows x heads, and of 16 new tokens)
constexpr int64_t kMostGroups = int64_t(1) << 24;
// The kernels count places of a sequence in 32 bits: those of its table and behind them the 16 of each unit that a launch may have (and with them all new tokens, fewer
// than 2^28).
constexpr int32_t kMostTablePages = (1 << 27) - (1 << 24) - 1;
inline bool batch_ok(const card_model_cfg* cfg, const card_kv_batch* b) {
    return cfg_valid(cfg) && b && b->n_pages > 0 && b->n_seqs > 0 && b->table_pages > 0 && b->table_pages <= kMostTablePages && b->n_rows >= 0 &&
           b->max_new >= 0 && b->max_len >= 0;
}
inline bool batch_fits(const card_model_cfg* cfg, const card_kv_batch* b) {
    return int64_t(b->n_rows) * cfg->n_q_heads / 16 + int64_t(kStoreUnits) * b->n_seqs * cfg->n_kv_heads < kMostGroups;
}

struct AttendPlan {
    int32_t tiles, units, cuts, cut_pages;
    bool fused;
    size_t bytes;
};

inline int layer_refused(const card_model_cfg* cfg, const card_kv_batch* batch, int32_t layer) {
    if (!batch_ok(cfg, batch)) return CARD_EINVAL;
    if (!batch->k_pages || !batch->v_pages || !batch->block_tables || !batch->ctx_lens || !batch->row_starts) return CARD_EINVAL;
    if (!aligned16(batch->k_pages) || !aligned16(batch->v_pages)) return CARD_EINVAL;
    if (layer < 0 || layer >= cfg->n_layers) return CARD_ERANGE;
    return batch_fits(cfg, batch) ? CARD_OK : CARD_ERANGE;
}
inline int attend_refused(const card_model_cfg* cfg, const card_kv_batch* batch, int32_t layer, const card_rows* q, const card_rows* k, const card_rows* v,
                   const card_rows* out, const card_row_mask* mask) {
    if (const int st = layer_refused(cfg, batch, layer)) return st;
    if (batch->n_rows == 0) return CARD_OK;
    if (!q || !out || (q->type != CARD_BF16 && q->type != CARD_F32)) return CARD_EINVAL;
    if (!rows_ok(q, q->type, 0) || !rows_ok(out, q->type, cfg->head_dim) || !k != !v) return CARD_EINVAL;
    if (k && (!rows_ok(k, q->type, 0) || !rows_ok(v, q->type, 0))) return CARD_EINVAL;
    if (mask && (!mask->mask_dev || !mask->mask_base_dev || mask->words < 1 || mask->words > (1 << 25))) return CARD_EINVAL;
    return CARD_OK;
}

// bits: of a value in the cache, 16 or 4.  Without a plan, what storing needs.
inline AttendArgs attend_args(const card_model_cfg* cfg, const card_kv_batch* batch, int32_t layer, int bits, const card_rows* q, const card_rows* k,
                       const card_rows* v, const card_rows* out, const card_row_mask* mask, const AttendPlan& plan, void* workspace_dev) {
    AttendArgs a = {};
    if (q) {
        a.q = q->data;
        a.q_row = q->row_stride;
        a.q_head = q->head_stride;
        a.out = out->data;
        a.o_row = out->row_stride;
        a.o_head = out->head_stride;
    }
    if (k) {
        a.k = k->data;
        a.k_row = k->row_stride;
        a.k_head = k->head_stride;
        a.v = v->data;
        a.v_row = v->row_stride;
        a.v_head = v->head_stride;
    }
    const size_t before = size_t(layer) * layer_bytes(cfg, batch->n_pages, bits);
    a.kpool = reinterpret_cast<__bf16*>(static_cast<char*>(batch->k_pages) + before);
    a.vpool = reinterpret_cast<__bf16*>(static_cast<char*>(batch->v_pages) + before);
    a.tables = batch->block_tables;
    a.ctx = batch->ctx_lens;
    a.starts = batch->row_starts;
    a.table_pages = batch->table_pages;
    a.n_pages = batch->n_pages;
    a.n_seqs = batch->n_seqs;
    a.n_rows = batch->n_rows;
    a.Hkv = cfg->n_kv_heads;
    a.G = cfg->n_q_heads / cfg->n_kv_heads;
    if (mask) {
        a.mask = mask->mask_dev;
        a.mask_base = mask->mask_base_dev;
        a.mask_words = mask->words;
    }
    a.scale = 1.4426950408889634f / sqrtf(float(cfg->head_dim));
    a.cuts = plan.cuts;
    a.cut_pages = plan.cut_pages;
    a.part = static_cast<float*>(workspace_dev);
    return a;
}

// How a row of logits is cut: one workgroup per row where the rows fill the GPU, else parts of 4096 logits or more (one row of 128256 in fp32 in parts
// of 1024, 4096, 16384 or whole 9.5, 9.2, 12.2, 26 us, eight 10.2, 9.3, 13.0, 28).  1000 rows of 152064 in bf16,
// the most probable token: for 512, 768, 1024 or 2048 workgroups 54.7, 55.1, 59.4, 67.4 us; 300 rows 28.6, 27.6, 26.8, 30.1; 100 of 128256 in fp32
// 16.5, 15.8, 15.8, 17.7.
inline int32_t logprob_parts(int32_t rows, int32_t vocab) { return std::min(ceil_div(vocab, 4096), ceil_div(768, rows)); }
constexpr int32_t kMostLogits = 1 << 30;  // of a row: they are counted in 32 bits, with the rest of a 16-byte unit at either end
inline size_t logprob_sums_bytes(int32_t rows, int32_t vocab) { return size_t(rows) * logprob_parts(rows, vocab) * 16; }

}  // namespace card
