// Selection of beams: of each group of them, the best continuations over beams and vocabulary.
//
// A candidate's score is its beam's score + (x - m) / T - ln s, with m the beam's largest logit and s = sum e^((x - m) / T): inside a beam the order of scores is that of the
// logits, so of each beam only its most probable tokens matter, as many as there are beams to go on with.  One pass over the logits finds them with m and s
// (scan_part), and bounds it: LISTED.  Scores of several beams are compared in 64 bits, so that sums of hundreds of log probabilities do not hide what
// the candidates differ by.
#pragma once
#include "card_logprobs.hip"

namespace card {

constexpr int kMostBeams = 32;

struct BeamArgs {
    LogprobArgs rows;  // (top: beams to go on with)
    int32_t beams, eos, history_len;
    double temperature;
    const float* scores;
    const int32_t* done;
    const int32_t* history;
    const int32_t* lengths;
    float* out_scores;
    int32_t* out_tokens;
    int32_t* out_parents;
    int32_t* out_done;
    int32_t* out_history;
};

// One workgroup: one part of the logits of one beam.  Those of a beam that has ended are not read.
template <typename T>
__global__ __launch_bounds__(kLpThreads) void k_beam_rows(BeamArgs b) {
    __shared__ LogprobShared sm;
    const int row = blockIdx.x, part = blockIdx.y;
    if (b.done && b.done[row] != 0) return;
    const RowSums r = scan_part<T>(b.rows, sm, row, part);
    leave_part(b.rows, sm, r, row, part);
}

// One workgroup: one group.  A wavefront puts the parts of a beam together; then a candidate's place is the number of better ones.  Candidates with equal scores
// go by beam, then by token; a beam's list has them in that order.
__global__ __launch_bounds__(1024) void k_beam_join(BeamArgs b) {
    __shared__ double score[kMostBeams * kMaxTop];
    __shared__ int token[kMostBeams * kMaxTop];
    __shared__ int parent_of[kMaxTop], token_of[kMaxTop];
    const LogprobArgs& a = b.rows;
    const int group = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6, top = a.top;
    const float c = a.inv_temp * kLog2e;
    for (int beam = wave; beam < b.beams; beam += waves) {
        const int row = group * b.beams + beam, n = a.parts * top;
        const double held = b.scores[row];
        const bool there = held > -INFINITY && held < INFINITY, ended = b.done && b.done[row] != 0;
        double mine = -INFINITY;
        int tok = -1;
        if (there && ended) {
            if (lane == 0) {
                mine = held;
                tok = b.eos;
            }
        } else if (there) {
            RowSums r = {kLowest, 0.f, 0.f};
            for (int p = lane; p < a.parts; p += 64) {
                const floatx4 v = *reinterpret_cast<const floatx4*>(a.part_sums + (size_t(row) * a.parts + p) * 4);
                r.join(RowSums{v[0], v[1], v[2]}, c);
            }
            r = join_lanes(r, c);
            TopList list;
            const unsigned long long* keys = a.part_keys + size_t(row) * n;
            if (a.parts >= top) list.floor(lane < a.parts ? uint32_t(keys[lane * top] >> 32) : 0u, top);  // of the parts' first keys, the top-th largest
            for (int i = 0; i < n; i += 64) list.offer(i + lane < n ? keys[i + lane] : 0ull, top, lane);
            // (a NaN or +inf among the logits has made s NaN: no candidates)
            if (lane < top && list.best != 0ull && r.s > 0.f) {
                mine = held + ((double(key_logit(list.best)) - double(r.m)) / b.temperature - log(double(r.s)));
                tok = int(0xffffffffu - uint32_t(list.best));
            }
        }
        if (lane < top) {
            score[beam * top + lane] = mine;
            token[beam * top + lane] = tok;
        }
    }
    if (tid < top) parent_of[tid] = -1;
    __syncthreads();
    const int all = b.beams * top;
    for (int i = tid; i < all; i += blockDim.x) {
        const double s = score[i];
        if (!(s > -INFINITY)) continue;
        int better = 0;
        for (int j = 0; j < all; ++j) better += score[j] > s || (score[j] == s && j < i);
        if (better >= top) continue;
        const int beam = i / top;
        const size_t to = size_t(group) * top + better;
        parent_of[better] = beam;
        token_of[better] = token[i];
        b.out_scores[to] = float(s);
        b.out_tokens[to] = token[i];
        b.out_parents[to] = beam;
        if (b.out_done) b.out_done[to] = (b.done && b.done[group * b.beams + beam] != 0) || (b.eos >= 0 && token[i] == b.eos);
    }
    __syncthreads();
    if (tid < top && parent_of[tid] < 0) {  // fewer candidates than that
        const size_t to = size_t(group) * top + tid;
        b.out_scores[to] = -INFINITY;
        b.out_tokens[to] = -1;
        b.out_parents[to] = 0;
        if (b.out_done) b.out_done[to] = 1;
    }
    if (!b.history) return;
    const int len = min(max(b.lengths[group], 0), b.history_len);
    for (int k = 0; k < top; ++k) {
        if (parent_of[k] < 0) continue;
        const int32_t* from = b.history + (size_t(group) * b.beams + parent_of[k]) * b.history_len;
        int32_t* to = b.out_history + (size_t(group) * top + k) * b.history_len;
        for (int i = tid; i < len; i += blockDim.x) to[i] = from[i];
        if (tid == 0 && len < b.history_len) to[len] = token_of[k];
    }
}

}  // namespace card
