// C ABI of what serves several sequences from one pair of page pools: argument checks and launches of page copies, slot
// moves, attention over a ragged batch and log probabilities.
#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <hip/hip_runtime.h>

#include "card.h"
#include "card_attend.hip"
#include "card_logprobs.hip"
#include "card_pages.hip"

using namespace card;

namespace {

inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
inline int launch_status() { return hipGetLastError() == hipSuccess ? CARD_OK : CARD_EDEVICE; }
inline bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
inline size_t layer_elems(const card_model_cfg* cfg, int32_t n_pages) { return size_t(n_pages) * cfg->n_kv_heads * 16 * cfg->head_dim; }

// A set of numbers >= 0, open addressing.
class NumberSet {
public:
    explicit NumberSet(int32_t n) {
        for (; size_ < 2 * size_t(n); size_ *= 2) --shift_;
        at_ = static_cast<int32_t*>(malloc(size_ * sizeof(int32_t)));
        if (at_) std::fill(at_, at_ + size_, -1);
    }
    ~NumberSet() { free(at_); }
    NumberSet(const NumberSet&) = delete;
    NumberSet& operator=(const NumberSet&) = delete;
    bool ok() const { return at_ != nullptr; }
    bool has(int32_t v) const { return at_[place(v)] == v; }
    bool add(int32_t v) {  // false: it was there
        int32_t& p = at_[place(v)];
        if (p == v) return false;
        p = v;
        return true;
    }

private:
    size_t place(int32_t v) const {
        size_t i = (uint32_t(v) * 0x9e3779b1u) >> shift_;  // the upper bits: numbers that lie a power of two apart spread, too
        while (at_[i] != -1 && at_[i] != v) i = (i + 1) & (size_ - 1);
        return i;
    }
    size_t size_ = 16;
    int shift_ = 28;  // 32 - log2(size_)
    int32_t* at_ = nullptr;
};

int pool_args(const card_model_cfg* cfg, const card_kv* kv, int32_t n, const int32_t* src, const int32_t* dst) {
    if (!cfg_valid(cfg) || !kv || !kv->k_pages || !kv->v_pages || kv->n_pages <= 0 || n < 0) return CARD_EINVAL;
    if (n > 0 && (!src || !dst)) return CARD_EINVAL;
    if (!aligned16(kv->k_pages) || !aligned16(kv->v_pages)) return CARD_EINVAL;
    return CARD_OK;
}

bool rows_ok(const card_rows* r, int32_t type, int64_t least_stride) {
    const int64_t unit = type == CARD_F32 ? 4 : 8;
    return r && r->data && r->type == type && aligned16(r->data) && r->row_stride >= least_stride && r->head_stride >= least_stride &&
           r->row_stride % unit == 0 && r->head_stride % unit == 0;
}

bool batch_ok(const card_model_cfg* cfg, const card_kv_batch* b) {
    return cfg_valid(cfg) && b && b->n_pages > 0 && b->n_seqs > 0 && b->table_pages > 0 && b->table_pages < (1 << 27) && b->n_rows >= 0 &&
           b->max_new >= 0 && b->max_len >= 0;
}

// A launch has less than 2^32 threads in x: 2^24 workgroups of 256.  (units of 16 rows x heads, and of 16 new tokens)
constexpr int64_t kMostGroups = int64_t(1) << 24;
bool batch_fits(const card_model_cfg* cfg, const card_kv_batch* b) {
    return int64_t(b->n_rows) * cfg->n_q_heads / 16 + int64_t(kStoreUnits) * b->n_seqs * cfg->n_kv_heads < kMostGroups;
}

template <int ROUND>
void move_launch(const MoveArgs& a, int h, dim3 grid, hipStream_t st) {
    if (h == 128) hipLaunchKernelGGL((k_kv_move_slots<128, ROUND>), grid, dim3(384), 0, st, a);
    else hipLaunchKernelGGL((k_kv_move_slots<64, ROUND>), grid, dim3(192), 0, st, a);
}

// How a row of logits is cut: one workgroup per row where the rows fill the GPU, else parts of 4096 logits or more (one row of 128256 in fp32 in parts
// of 1024, 4096, 16384 or whole 9.5, 9.2, 12.2, 26 us, eight 10.2, 9.3, 13.0, 28).  1000 rows of 152064 in bf16,
// the most probable token: for 512, 768, 1024 or 2048 workgroups 54.7, 55.1, 59.4, 67.4 us; 300 rows 28.6, 27.6, 26.8, 30.1; 100 of 128256 in fp32
// 16.5, 15.8, 15.8, 17.7.
int32_t logprob_parts(int32_t rows, int32_t vocab) { return std::min(ceil_div(vocab, 4096), ceil_div(768, rows)); }
constexpr int32_t kMostLogits = 1 << 30;  // of a row: they are counted in 32 bits, with the rest of a 16-byte unit at either end
size_t logprob_sums_bytes(int32_t rows, int32_t vocab) { return size_t(rows) * logprob_parts(rows, vocab) * 16; }

template <typename T>
int logprobs_launch(const LogprobArgs& a, int32_t rows, hipStream_t st) {
    hipLaunchKernelGGL(k_logprobs<T>, dim3(uint32_t(rows), uint32_t(a.parts)), dim3(kLpThreads), 0, st, a);
    if (a.parts > 1) hipLaunchKernelGGL(k_logprobs_join<T>, dim3(uint32_t(rows)), dim3(kLpThreads), 0, st, a);
    return launch_status();
}

// How the attention of a call is run.  R: most rows x heads of a KV head that one sequence has; all figures in us, 8 KV heads of 128.
// Tiles of 16 rows x heads of a workgroup.  R <= 16 one: R = 16 of 16 texts of 300-3000 tokens 25.8, with two 33.0.  R <= 512 two, which
// read the cache half as often: R = 64 of 48 texts of 400-4000 tokens 117, with one 134.  Above, k_attend_many.  Two tiles and k_attend_many, R = 384, 512, 768: a
// text of 14000 tokens 55 and 57, 70 and 67, 108 and 87; of 300 tokens 13 and 18, 13 and 22, 13 and 24; 16 texts of 300-3000 71 and 80, 85 and 98, 119 and
// 137; 48 of 100-1000 86 and 91, 109 and 109, 154 and 138.  fp32: one, whose three parts of a row fill the registers as more rows would (R = 256: 73,
// with two 101).
// The new tokens are stored by the same kernel as long as R <= 256 and they have room in LDS, else by one in front: R = 32 of one text 20.3
// and 23.0, R = 256 40.6 and 42.7, R = 384 of 16 texts 80 and 71, R = 512 of 48 151 and 109.
constexpr int kFewRows = 512, kFewStore = 256;
// The pages of a sequence are cut to have this many workgroups, two per compute unit, unless there are three quarters of them
// without (one token each, 256, 512, 768, 2048 workgroups: a text of 14000 tokens 16.1, 18.3, 18.3, 21.4; 48 texts of 400-4000 94.3, 94.2, 93.5, 99.6; R = 128,
// 14000 tokens, 256, 512, 768: 35, 28, 33; k_attend_many, 250 tokens behind 14000: 121, 98, 115).  Counted by rows, so that texts of a few rows, which
// differ in length, are cut more than that: 48 texts in five cuts 94.2, in two (768 workgroups) 99.6.
constexpr int kFill = 512;
// Cuts cost the join, 3 us and a share per workgroup, and gain where a workgroup's pages take longer: not for so many pages.  (uncut and cut; one token each: a
// text of 500 tokens 7.6 and 8.4, 1000 11.0 and 8.4; 8 texts of 1000 11.1 and 10.1; 30 of 1000 17.6 and 19.4, of 1500 23.5 and 24.3; 100 of 2000 99 and
// 100; R = 512 behind 700 tokens 16.5 and 18.2, behind 2000 28.0 and 23.6; k_attend_many, R = 640 behind 100 17.9 and 18.9, behind 700 34 and 24, R = 2000 behind 300 33 and
// 33, behind 500 39 and 35, behind 1500 67 and 46, R = 4000 behind 1000 69 and 71.)
int64_t pages_uncut(int tiles, int64_t groups) { return tiles == kManyTiles ? 8 + groups / 2 : 32 + groups / 3; }
struct AttendPlan {
    int32_t tiles, units, cuts, cut_pages;
    bool fused;
    size_t bytes;
};
AttendPlan attend_plan(const card_model_cfg* cfg, const card_kv_batch* b, bool f32) {
    AttendPlan p = {};
    const int G = cfg->n_q_heads / cfg->n_kv_heads;
    const int64_t most = int64_t(b->max_new > 0 ? std::min(b->max_new, b->n_rows) : b->n_rows) * G;
    p.fused = most <= std::min(kFewStore, kStage * G);
    p.tiles = f32 || most <= 16 ? 1 : (most <= kFewRows ? 2 : kManyTiles);
    p.units = int32_t(int64_t(b->n_rows) * G / (16 * p.tiles)) + b->n_seqs;
    const int pages = std::min(b->table_pages, b->max_len > 0 ? ceil_div(b->max_len, 16) : b->table_pages);
    const int full = p.units - b->n_seqs + 1;  // tiles, if the rows filled them
    const int64_t groups = int64_t(full) * cfg->n_kv_heads;
    const bool whole = groups * 4 > kFill * 3 || pages <= pages_uncut(p.tiles, int64_t(std::max(full, b->n_seqs)) * cfg->n_kv_heads);
    p.cut_pages = whole ? pages : std::max(8, ceil_div(ceil_div(groups * pages, kFill), 8) * 8);
    p.cuts = ceil_div(pages, p.cut_pages);
    if (p.cuts > 1) p.bytes = size_t(p.units) * cfg->n_kv_heads * p.cuts * p.tiles * 16 * (cfg->head_dim + 2) * 4;
    return p;
}

template <int H, typename T, int NT>
void attend_launch(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
    const dim3 grid(uint32_t(p.units) * uint32_t(a.Hkv), uint32_t(p.cuts));
    if (a.k && !p.fused)
        hipLaunchKernelGGL((k_attend_store<H, T>), dim3(uint32_t(a.n_rows / 16 + kStoreUnits * a.n_seqs), uint32_t(a.Hkv)), dim3(256), 0, st, a);
    if constexpr (NT == kManyTiles) hipLaunchKernelGGL(k_attend_many<H>, grid, dim3(256), 0, st, a);
    else if (a.k && p.fused) hipLaunchKernelGGL((k_attend_few<H, T, NT, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_attend_few<H, T, NT, false>), grid, dim3(256), 0, st, a);
    if (p.cuts > 1) hipLaunchKernelGGL((k_attend_join<H, T, NT>), dim3(grid.x, 4 * NT), dim3(256), 0, st, a);
}
template <typename T, int NT>
void attend_launch(const AttendArgs& a, const AttendPlan& p, int h, hipStream_t st) {
    h == 128 ? attend_launch<128, T, NT>(a, p, st) : attend_launch<64, T, NT>(a, p, st);
}

}  // namespace

extern "C" {

int card_kv_copy_pages(const card_model_cfg* cfg, const card_kv* kv, int32_t n, const int32_t* src_host, const int32_t* dst_host,
                       void* stream) {
    if (const int st = pool_args(cfg, kv, n, src_host, dst_host)) return st;
    if (n == 0) return CARD_OK;
    NumberSet written(n);
    if (!written.ok()) return CARD_EDEVICE;
    for (int i = 0; i < n; ++i) {
        if (src_host[i] < 0 || src_host[i] >= kv->n_pages || dst_host[i] < 0 || dst_host[i] >= kv->n_pages) return CARD_ERANGE;
        if (!written.add(dst_host[i])) return CARD_EINVAL;
    }
    for (int i = 0; i < n; ++i)
        if (written.has(src_host[i])) return CARD_EINVAL;
    CopyArgs a = {};
    a.pool[0] = static_cast<uint4v*>(kv->k_pages);
    a.pool[1] = static_cast<uint4v*>(kv->v_pages);
    a.layer16 = layer_elems(cfg, kv->n_pages) / 8;
    a.page16 = cfg->n_kv_heads * 2 * cfg->head_dim;
    for (int i = 0; i < n; i += kCopyPairs) {
        const int m = std::min(n - i, kCopyPairs);
        std::copy(src_host + i, src_host + i + m, a.src);
        std::copy(dst_host + i, dst_host + i + m, a.dst);
        hipLaunchKernelGGL(k_kv_copy_pages, dim3(uint32_t(m), uint32_t(cfg->n_layers), 2), dim3(256), 0, as_stream(stream), a);
    }
    return launch_status();
}

int card_kv_move_slots(const card_model_cfg* cfg, const card_kv* kv, int32_t n, const int32_t* src_host, const int32_t* dst_host,
                       void* stream) {
    if (const int st = pool_args(cfg, kv, n, src_host, dst_host)) return st;
    if (n == 0) return CARD_OK;
    NumberSet written(n);
    if (!written.ok()) return CARD_EDEVICE;
    const int64_t slots = int64_t(kv->n_pages) * 16;
    for (int i = 0; i < n; ++i) {
        if (src_host[i] < 0 || src_host[i] >= slots || dst_host[i] < 0 || dst_host[i] >= slots) return CARD_ERANGE;
        if (written.has(src_host[i]) || !written.add(dst_host[i])) return CARD_EINVAL;
    }
    bool apart = true;  // no move writes what another one reads: they need no order
    for (int i = 0; i < n; ++i) apart = apart && !written.has(src_host[i]);
    MoveArgs a = {};
    a.kpool = static_cast<__bf16*>(kv->k_pages);
    a.vpool = static_cast<__bf16*>(kv->v_pages);
    a.layer_elems = layer_elems(cfg, kv->n_pages);
    a.n_kv_heads = cfg->n_kv_heads;
    for (int i = 0; i < n;) {
        for (a.n = 0; i < n && a.n < kMoveSlots; ++a.n) {
            const int32_t* d = dst_host + i;
            const bool four = i + 4 <= n && d[1] == d[0] + 1 && d[2] == d[0] + 2 && d[3] == d[0] + 3;
            a.src[a.n] = src_host[i];
            a.dst[a.n] = four && (d[0] - a.n) % 4 != 0 ? -1 : d[0];
            i += a.dst[a.n] >= 0;
        }
        a.part = apart ? kMoveApart : kMoveSlots;
        const dim3 grid(uint32_t(cfg->n_kv_heads), uint32_t(cfg->n_layers), uint32_t(ceil_div(a.n, a.part)));
        if (apart || a.n <= 7 * kMoveShort) move_launch<kMoveShort>(a, cfg->head_dim, grid, as_stream(stream));
        else move_launch<kMoveRound>(a, cfg->head_dim, grid, as_stream(stream));
    }
    return launch_status();
}

size_t card_kv_attend_workspace_bytes(const card_model_cfg* cfg, const card_kv_batch* batch) {
    if (!batch_ok(cfg, batch) || !batch_fits(cfg, batch) || batch->n_rows == 0) return 0;
    return std::max(attend_plan(cfg, batch, false).bytes, attend_plan(cfg, batch, true).bytes);
}

int card_kv_attend(const card_model_cfg* cfg, const card_kv_batch* batch, int32_t layer, const card_rows* q, const card_rows* k,
                   const card_rows* v, const card_rows* out, const card_row_mask* mask, void* workspace_dev, void* stream) {
    if (!batch_ok(cfg, batch)) return CARD_EINVAL;
    if (!batch->k_pages || !batch->v_pages || !batch->block_tables || !batch->ctx_lens || !batch->row_starts) return CARD_EINVAL;
    if (!aligned16(batch->k_pages) || !aligned16(batch->v_pages)) return CARD_EINVAL;
    if (layer < 0 || layer >= cfg->n_layers) return CARD_ERANGE;
    if (!batch_fits(cfg, batch)) return CARD_ERANGE;
    if (batch->n_rows == 0) return CARD_OK;
    if (!q || !out || (q->type != CARD_BF16 && q->type != CARD_F32)) return CARD_EINVAL;
    if (!rows_ok(q, q->type, 0) || !rows_ok(out, q->type, cfg->head_dim) || !k != !v) return CARD_EINVAL;
    if (k && (!rows_ok(k, q->type, 0) || !rows_ok(v, q->type, 0))) return CARD_EINVAL;
    if (mask && (!mask->mask_dev || !mask->mask_base_dev || mask->words < 1 || mask->words > (1 << 25))) return CARD_EINVAL;
    const AttendPlan plan = attend_plan(cfg, batch, q->type == CARD_F32);
    if (plan.bytes > 0 && (!workspace_dev || !aligned16(workspace_dev))) return CARD_EINVAL;
    AttendArgs a = {};
    a.q = q->data;
    a.q_row = q->row_stride;
    a.q_head = q->head_stride;
    if (k) {
        a.k = k->data;
        a.k_row = k->row_stride;
        a.k_head = k->head_stride;
        a.v = v->data;
        a.v_row = v->row_stride;
        a.v_head = v->head_stride;
    }
    a.out = out->data;
    a.o_row = out->row_stride;
    a.o_head = out->head_stride;
    a.kpool = static_cast<__bf16*>(batch->k_pages) + size_t(layer) * layer_elems(cfg, batch->n_pages);
    a.vpool = static_cast<__bf16*>(batch->v_pages) + size_t(layer) * layer_elems(cfg, batch->n_pages);
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
    hipStream_t st = as_stream(stream);
    const int h = cfg->head_dim;
    if (q->type == CARD_F32) attend_launch<float, 1>(a, plan, h, st);
    else if (plan.tiles == 1) attend_launch<__bf16, 1>(a, plan, h, st);
    else if (plan.tiles == 2) attend_launch<__bf16, 2>(a, plan, h, st);
    else attend_launch<__bf16, kManyTiles>(a, plan, h, st);
    return launch_status();
}

size_t card_logprobs_workspace_bytes(int32_t rows, int32_t vocab, int32_t top) {
    if (rows < 1 || vocab < 1 || top < 0 || top > kMaxTop || ceil_div(vocab, 4096) == 1) return 0;
    // (r rows have at most r + 767 parts: enough for fewer rows, too)
    const int64_t parts = std::min(int64_t(rows) * ceil_div(vocab, 4096), int64_t(rows) + 768);
    return size_t(parts) * (16 + 8 * size_t(top));
}

int card_logprobs(const void* logits_dev, int32_t type, int32_t rows, int32_t vocab, int64_t row_stride, const int32_t* tokens_dev,
                  float temperature, int32_t top, float* logprob_dev, float* entropy_dev, int32_t* top_tokens_dev,
                  float* top_logprobs_dev, void* workspace_dev, void* stream) {
    if ((type != CARD_BF16 && type != CARD_F32) || rows < 0 || vocab < 1 || row_stride < vocab) return CARD_EINVAL;
    if (!(temperature >= 1e-30f && temperature <= 1e30f)) return CARD_EINVAL;
    if (top < 0 || top > kMaxTop || rows >= kMostGroups || vocab >= kMostLogits) return CARD_ERANGE;
    if (rows == 0) return CARD_OK;
    if (!logits_dev || !tokens_dev != !logprob_dev || (top > 0 && (!top_tokens_dev || !top_logprobs_dev))) return CARD_EINVAL;
    if (!tokens_dev && !entropy_dev && top == 0) return CARD_EINVAL;
    const int parts = logprob_parts(rows, vocab);
    if (parts > 1 && (!workspace_dev || !aligned16(workspace_dev))) return CARD_EINVAL;
    LogprobArgs a = {logits_dev,  row_stride,  vocab,          top,             tokens_dev, 1.0f / temperature,
                     logprob_dev, entropy_dev, top_tokens_dev, top_logprobs_dev};
    const int units = vocab / (type == CARD_F32 ? 4 : 8) + 2;  // of 16 bytes, the ends of a row that begins anywhere among them
    a.part_vecs = ceil_div(units, parts);
    a.parts = ceil_div(units, a.part_vecs);
    if (parts > 1) {
        a.part_sums = static_cast<float*>(workspace_dev);
        a.part_keys = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace_dev) + logprob_sums_bytes(rows, vocab));
    }
    return type == CARD_F32 ? logprobs_launch<float>(a, rows, as_stream(stream)) : logprobs_launch<__bf16>(a, rows, as_stream(stream));
}

}  // extern "C"
