// C ABI of rotation with storing, of the cache of 4 bits a value and of the selection of beams: argument checks and launches.
#include <algorithm>
#include <cmath>
#include <hip/hip_runtime.h>

#include "card.h"
#include "card_append.hip"
#include "card_attend4.hip"
#include "card_beams.hip"
#include "card_serving.h"

using namespace card;

namespace {

// How the attention of a call over 4 bits is run.  R: most rows x heads of a KV head that one sequence has; all figures in us, 8 KV heads of 128.
// Tiles of 16 rows x heads of a workgroup: one, in bf16 two for R > 1024 (R = 600 behind 3000 tokens 35 and 33, behind 14000 95 and 99; 2000 behind 300 22 and
// 23, behind 14000 284 and 258; 8000 behind 14000 1097 and 999; 40 behind 120000 73 and 84).  Making operands of codes is work that
// tiles share, and half as many wavefronts hide each other's waits.
constexpr int kOneTile4 = 1024;
// Pages are cut to have this many workgroups, three per compute unit, unless there are half of them without, counted by rows as in attend_plan (in cuts of 32, 64, 128, 256
// pages and uncut: 64 texts of 800-8000 tokens, one row each, 97, 86, 81, 87, 135; 48 of 400-4000 39, 38, 40, 61, 61; 16 of 300-3000 17, 20, 25, 36, 36; R = 400 behind 4000
// tokens 38, 32, 32, 38, 38; R = 600 behind 14000 126, 104, 100, 95, 163; R = 2000 behind 3000 105, 90, 84, 75, 75).
constexpr int kFill4 = 768, kLeastCut4 = 32;
// (uncut and in cuts of 32: one row of 1000 tokens 11.7 and 11.8, of 1500 15.7 and 12.0, of 3000 32 and 11; R = 400 behind 1000 13.0 and 15.8, in fp32 behind 1024 14.3 and 15.2)
int64_t pages_uncut4(int64_t groups) { return 64 + groups / 8; }
AttendPlan attend4_plan(const card_model_cfg* cfg, const card_kv_batch* b, bool f32) {
    AttendPlan p = {};
    const int G = cfg->n_q_heads / cfg->n_kv_heads;
    const int64_t most = int64_t(b->max_new > 0 ? std::min(b->max_new, b->n_rows) : b->n_rows) * G;
    p.tiles = f32 || most <= kOneTile4 ? 1 : 2;
    p.units = int32_t(int64_t(b->n_rows) * G / (16 * p.tiles)) + b->n_seqs;
    const int pages = std::min(b->table_pages, b->max_len > 0 ? ceil_div(b->max_len, 16) : b->table_pages);
    const int full = p.units - b->n_seqs + 1;  // tiles, if the rows filled them
    const int64_t groups = int64_t(full) * cfg->n_kv_heads;
    const bool whole = groups * 2 > kFill4 || pages <= pages_uncut4(int64_t(std::max(full, b->n_seqs)) * cfg->n_kv_heads);
    p.cut_pages = whole ? pages : std::max(kLeastCut4, ceil_div(ceil_div(groups * pages, kFill4), 16) * 16);
    p.cuts = ceil_div(pages, p.cut_pages);
    if (p.cuts > 1) p.bytes = size_t(p.units) * cfg->n_kv_heads * p.cuts * p.tiles * 16 * (cfg->head_dim + 2) * 4;
    return p;
}
template <int H, typename T>
void append_launch(const AppendArgs& g, int bits, hipStream_t st) {
    const dim3 grid(uint32_t(g.a.n_rows / 16 + kStoreUnits * g.a.n_seqs), uint32_t(g.a.Hkv));
    if (bits == 16) hipLaunchKernelGGL((k_append<H, T, 16>), grid, dim3(256), 0, st, g);
    else hipLaunchKernelGGL((k_append<H, T, 4>), grid, dim3(256), 0, st, g);
}
template <typename T>
void append_launch(const AppendArgs& g, int bits, int h, hipStream_t st) {
    h == 128 ? append_launch<128, T>(g, bits, st) : append_launch<64, T>(g, bits, st);
}
template <int H, typename T, int NT>
void attend4_launch(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
    const dim3 grid(uint32_t(p.units) * uint32_t(a.Hkv), uint32_t(p.cuts));
    hipLaunchKernelGGL((k_attend4<H, T, NT>), grid, dim3(256), 0, st, a);
    if (p.cuts > 1) hipLaunchKernelGGL((k_attend_join<H, T, NT>), dim3(grid.x, 4 * NT), dim3(256), 0, st, a);
}
template <typename T, int NT>
void attend4_launch(const AttendArgs& a, const AttendPlan& p, int h, hipStream_t st) {
    h == 128 ? attend4_launch<128, T, NT>(a, p, st) : attend4_launch<64, T, NT>(a, p, st);
}

constexpr int kHistoryShare = 1024;  // of a workgroup of k_beam_join (tokens)

int append(const card_model_cfg* cfg, const card_kv_batch* batch, int32_t layer, int bits, const card_rotation* rotation, const card_rows* q,
           const card_rows* q_out, const card_rows* k, const card_rows* v, void* stream) {
    if (const int st = layer_refused(cfg, batch, layer)) return st;
    if (batch->n_rows == 0) return CARD_OK;
    if (!k || !v || (k->type != CARD_BF16 && k->type != CARD_F32) || !rows_ok(k, k->type, 0) || !rows_ok(v, k->type, 0)) return CARD_EINVAL;
    if (!q != !q_out || (q && !rotation)) return CARD_EINVAL;
    if (q && (!rows_ok(q, k->type, 0) || !rows_ok(q_out, k->type, cfg->head_dim))) return CARD_EINVAL;
    const int h = cfg->head_dim;
    AppendArgs g = {};
    g.a = attend_args(cfg, batch, layer, bits, q, k, v, q_out, nullptr, AttendPlan{}, nullptr);
    if (rotation) {
        g.rotate = 1;
        g.positions = rotation->positions_dev;
        double near[8], far[8];  // powers of the base: a call takes 16 of them, not 64
        for (int i = 0; i < 8 && !rotation->freqs_host; ++i) {
            near[i] = std::pow(double(cfg->rope_theta), -2.0 * i / h);
            far[i] = std::pow(double(cfg->rope_theta), -16.0 * i / h);
        }
        for (int j = 0; j < h / 2; ++j) {
            const double f = rotation->freqs_host ? rotation->freqs_host[j] : near[j % 8] * far[j / 8];
            if (!std::isfinite(f)) return CARD_EINVAL;
            g.turns[j] = f / 6.283185307179586476925;
        }
    }
    k->type == CARD_F32 ? append_launch<float>(g, bits, h, as_stream(stream)) : append_launch<__bf16>(g, bits, h, as_stream(stream));
    return launch_status();
}

}  // namespace

extern "C" {

int card_kv_append(const card_model_cfg* cfg, const card_kv_batch* batch, int32_t layer, const card_rotation* rotation, const card_rows* q,
                   const card_rows* q_out, const card_rows* k, const card_rows* v, void* stream) {
    return append(cfg, batch, layer, 16, rotation, q, q_out, k, v, stream);
}

size_t card_kv4_pool_bytes(const card_model_cfg* cfg, int32_t n_pages) {
    return cfg_valid(cfg) && n_pages > 0 ? size_t(cfg->n_layers) * layer_bytes(cfg, n_pages, 4) : 0;
}

int card_kv4_append(const card_model_cfg* cfg, const card_kv_batch* batch, int32_t layer, const card_rotation* rotation, const card_rows* q,
                    const card_rows* q_out, const card_rows* k, const card_rows* v, void* stream) {
    return append(cfg, batch, layer, 4, rotation, q, q_out, k, v, stream);
}

int card_kv4_read(const card_model_cfg* cfg, const card_kv_batch* batch, int32_t layer, const card_rows* k, const card_rows* v, void* stream) {
    if (const int st = layer_refused(cfg, batch, layer)) return st;
    if (batch->n_rows == 0) return CARD_OK;
    const int h = cfg->head_dim;
    if (!k || !v || (k->type != CARD_BF16 && k->type != CARD_F32) || !rows_ok(k, k->type, h) || !rows_ok(v, k->type, h)) return CARD_EINVAL;
    const AttendArgs a = attend_args(cfg, batch, layer, 4, nullptr, k, v, nullptr, nullptr, AttendPlan{}, nullptr);
    const dim3 grid(uint32_t(a.n_rows / 16 + kStoreUnits * a.n_seqs), uint32_t(a.Hkv));
    hipStream_t st = as_stream(stream);
    if (k->type == CARD_F32 && h == 128) hipLaunchKernelGGL((k_read4<128, float>), grid, dim3(256), 0, st, a);
    else if (k->type == CARD_F32) hipLaunchKernelGGL((k_read4<64, float>), grid, dim3(256), 0, st, a);
    else if (h == 128) hipLaunchKernelGGL((k_read4<128, __bf16>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_read4<64, __bf16>), grid, dim3(256), 0, st, a);
    return launch_status();
}

size_t card_kv4_attend_workspace_bytes(const card_model_cfg* cfg, const card_kv_batch* batch) {
    if (!batch_ok(cfg, batch) || !batch_fits(cfg, batch) || batch->n_rows == 0) return 0;
    return std::max(attend4_plan(cfg, batch, false).bytes, attend4_plan(cfg, batch, true).bytes);
}

int card_kv4_attend(const card_model_cfg* cfg, const card_kv_batch* batch, int32_t layer, const card_rows* q, const card_rows* k,
                    const card_rows* v, const card_rows* out, const card_row_mask* mask, void* workspace_dev, void* stream) {
    if (const int st = attend_refused(cfg, batch, layer, q, k, v, out, mask)) return st;
    if (batch->n_rows == 0) return CARD_OK;
    const AttendPlan plan = attend4_plan(cfg, batch, q->type == CARD_F32);
    if (plan.bytes > 0 && (!workspace_dev || !aligned16(workspace_dev))) return CARD_EINVAL;
    if (k)
        if (const int st = append(cfg, batch, layer, 4, nullptr, nullptr, nullptr, k, v, stream)) return st;
    const AttendArgs a = attend_args(cfg, batch, layer, 4, q, nullptr, nullptr, out, mask, plan, workspace_dev);
    hipStream_t st = as_stream(stream);
    const int h = cfg->head_dim;
    if (q->type == CARD_F32) attend4_launch<float, 1>(a, plan, h, st);
    else if (plan.tiles == 1) attend4_launch<__bf16, 1>(a, plan, h, st);
    else attend4_launch<__bf16, 2>(a, plan, h, st);
    return launch_status();
}

size_t card_beam_select_workspace_bytes(int32_t groups, int32_t beams, int32_t out_beams, int32_t vocab) {
    if (groups < 1 || beams < 1 || beams > kMostBeams || out_beams < 1 || out_beams > kMaxTop || vocab < 1 || vocab >= kMostLogits) return 0;
    if (int64_t(groups) * beams >= kMostGroups) return 0;
    // (r rows have at most r + 767 parts: enough for fewer groups, too)
    const int64_t rows = int64_t(groups) * beams, parts = std::min(rows * ceil_div(vocab, 4096), rows + 768);
    return size_t(parts) * (16 + 8 * size_t(out_beams));
}

int card_beam_select(const void* logits_dev, int32_t type, int32_t vocab, int64_t row_stride, const card_beams* beams, float temperature,
                     void* workspace_dev, void* stream) {
    if (!beams || (type != CARD_BF16 && type != CARD_F32) || vocab < 1 || row_stride < vocab) return CARD_EINVAL;
    if (!(temperature >= 1e-30f && temperature <= 1e30f)) return CARD_EINVAL;
    if (beams->groups < 0 || beams->history_len < 0) return CARD_EINVAL;
    if (beams->beams < 1 || beams->beams > kMostBeams || beams->out_beams < 1 || beams->out_beams > kMaxTop || vocab >= kMostLogits) return CARD_ERANGE;
    if (int64_t(beams->groups) * beams->beams >= kMostGroups || beams->eos_token < -1 || beams->eos_token >= vocab) return CARD_ERANGE;
    if (beams->groups == 0) return CARD_OK;
    if (!logits_dev || !beams->scores_dev || !beams->out_scores_dev || !beams->out_tokens_dev || !beams->out_parents_dev) return CARD_EINVAL;
    if (beams->history_dev && (!beams->lengths_dev || !beams->out_history_dev)) return CARD_EINVAL;
    if (!workspace_dev || !aligned16(workspace_dev)) return CARD_EINVAL;
    const int rows = beams->groups * beams->beams, parts = logprob_parts(rows, vocab);
    BeamArgs b = {};
    LogprobArgs& a = b.rows;
    a.logits = logits_dev;
    a.row_stride = row_stride;
    a.vocab = vocab;
    a.top = beams->out_beams;
    a.inv_temp = 1.0f / temperature;
    const int units = vocab / (type == CARD_F32 ? 4 : 8) + 2;  // of 16 bytes, the ends of a row that begins anywhere among them
    a.part_vecs = ceil_div(units, parts);
    a.parts = ceil_div(units, a.part_vecs);
    a.part_sums = static_cast<float*>(workspace_dev);
    a.part_keys = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace_dev) + size_t(rows) * parts * 16);
    b.beams = beams->beams;
    b.eos = beams->eos_token;
    b.history_len = beams->history_len;
    b.temperature = temperature;
    b.scores = beams->scores_dev;
    b.done = beams->done_dev;
    b.history = beams->history_len > 0 ? beams->history_dev : nullptr;
    b.lengths = beams->lengths_dev;
    b.out_scores = beams->out_scores_dev;
    b.out_tokens = beams->out_tokens_dev;
    b.out_parents = beams->out_parents_dev;
    b.out_done = beams->out_done_dev;
    b.out_history = beams->out_history_dev;
    const dim3 grid(static_cast<uint32_t>(rows), uint32_t(a.parts));
    hipStream_t st = as_stream(stream);
    if (type == CARD_F32) hipLaunchKernelGGL(k_beam_rows<float>, grid, dim3(kLpThreads), 0, st, b);
    else hipLaunchKernelGGL(k_beam_rows<__bf16>, grid, dim3(kLpThreads), 0, st, b);
    const int64_t moved = b.history ? int64_t(b.history_len) * a.top : 0;
    const uint32_t shares = uint32_t(std::max(int64_t(1), std::min(int64_t(a.top), moved / kHistoryShare)));
    hipLaunchKernelGGL(k_beam_join, dim3(uint32_t(beams->groups), shares), dim3(64 * uint32_t(std::min(std::max(beams->beams, 4), 16))), 0, st, b);
    return launch_status();
}

}  // extern "C"
