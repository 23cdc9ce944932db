// Selection of beams: of each group of them, the best continuations over beams and vocabulary.
//
// A candidate's score is its beam's score + (x - m) / T - ln s, with m the beam's largest logit and s = sum e^((x - m) / T): inside a beam the order of scores is that of the
// logits, so of each beam only its most probable tokens matter, as many as there are beams to go on with.  One pass over the logits finds them with m and s
// (scan_part): 40 searches of 6 beams, 152064 tokens in bf16, an eighth of the beams ended, so 64 MB, in 23.2 us (2.8 TB/s), then 7.7 to join them; a search of 4 of 128256 in fp32
// 5.7 + 6.8.  The first is short rather than bound by one thing: 840 workgroups, one wave of them, vector units busy 43 % of the time (an exponential and some eight more instructions a
// logit), wavefronts waiting 58 %; 1000 rows go through the same pass at 5.2 TB/s.  The small ones are bound by latency.  Scores of several beams are compared in 64 bits, so that sums of hundreds of log probabilities do not hide what
// the candidates differ by.
#pragma once
#include "card_logprobs.hip"

namespace card {

constexpr int kMostBeams = 32;
constexpr int kHistoryLoads = 4;  // of a thread, under way together

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
    const RowSums r = scan_part<T, false, true>(b.rows, sm, row, part);
    leave_part(b.rows, sm, r, row, part);
}

__device__ __forceinline__ float first_lane(float v) { return __uint_as_float(uint32_t(__builtin_amdgcn_readfirstlane(int(__float_as_uint(v))))); }
// Scores as numbers in the same order (-0 as 0); 0: none.
__device__ __forceinline__ unsigned long long score_key(double s) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, s + 0.0);
    return s > -INFINITY ? (u >> 63 ? ~u : u | 1ull << 63) : 0ull;
}
__device__ __forceinline__ unsigned long long max_of_lanes(unsigned long long v) {
    v = group_max<16>(v);
    unsigned long long most = lane_key(v, 0);
#pragma unroll
    for (int row = 16; row < 64; row += 16) {
        const unsigned long long other = lane_key(v, row);
        most = other > most ? other : most;
    }
    return most;
}

// One workgroup: one group, or where histories are long a share of its new beams, which are chosen again by each.  A wavefront puts the parts of a beam together; then one
// wavefront, a beam a lane, takes the best of the lists' heads as often as there are beams to go on with, or ranks short lists at once.  Candidates with equal scores go by beam, then by token; a beam's list
// has them in that order.
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
            // (one lane's, for all: each adds up in another order, and equal logits are to have equal scores)
            const float most = first_lane(r.m), total = first_lane(r.s);
            TopList list;
            const unsigned long long* keys = a.part_keys + size_t(row) * n;
            if (n <= 64) {
                const unsigned long long key = lane < n ? keys[lane] : 0ull;
                if (a.parts > 3) list.floor(uint32_t(key >> 32), top);
                list.offer(key, top, lane);
            } else {  // rank by rank over the parts, whose lists are in order: where none of a rank enters, none behind it does
                for (int i = 0; i < n; i += 64) {
                    const uint32_t at = uint32_t(i + lane), parts = uint32_t(a.parts);
                    const unsigned long long key = at < uint32_t(n) ? keys[at % parts * top + at / parts] : 0ull;
                    if (i == 0) list.floor(uint32_t(key >> 32), top);
                    if (i > 0 && a.parts <= 64 && !__ballot(key > list.least)) break;
                    list.offer(key, top, lane);
                }
            }
            // (a NaN or +inf among the logits has made s NaN: no candidates)
            if (lane < top && list.best != 0ull && total > 0.f) {
                mine = held + ((double(key_logit(list.best)) - double(most)) / b.temperature - log(double(total)));
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
    const auto take = [&](int k, int i) {  // entry i of the lists is new beam k
        const int beam = i / top;
        parent_of[k] = beam;
        token_of[k] = token[i];
        if (blockIdx.y > 0) return;
        const size_t to = size_t(group) * top + k;
        b.out_scores[to] = float(score[i]);
        b.out_tokens[to] = token[i];
        b.out_parents[to] = beam;
        if (b.out_done) b.out_done[to] = (b.done && b.done[group * b.beams + beam] != 0) || (b.eos >= 0 && token[i] == b.eos);
    };
    const int all = b.beams * top;
    if (wave == 0 && all <= 64) {  // a lane each: its place is the number of better ones (a search of 4 beams 6.0 us, taken one by one 7.8)
        const unsigned long long mine = lane < all ? score_key(score[lane]) : 0ull;
        int better = 0;
        for (int j = 0; j < all; ++j) {
            const unsigned long long other = lane_key(mine, j);
            better += other > mine || (other == mine && j < lane);
        }
        if (mine != 0ull && better < top) take(better, lane);
    } else if (wave == 0) {
        int at = lane * top, left = lane < b.beams ? top : 0;
        unsigned long long head = left > 0 ? score_key(score[at]) : 0ull, next = left > 1 ? score_key(score[at + 1]) : 0ull;
        for (int k = 0; k < top; ++k) {
            const unsigned long long best = max_of_lanes(head);
            if (best == 0ull) break;
            if (lane != __ffsll(__ballot(head == best)) - 1) continue;
            take(k, at);
            head = next;
            ++at;
            --left;
            next = left > 1 ? score_key(score[at + 1]) : 0ull;
        }
    }
    __syncthreads();
    if (blockIdx.y == 0 && tid < top && parent_of[tid] < 0) {  // fewer candidates than that
        const size_t to = size_t(group) * top + tid;
        b.out_scores[to] = -INFINITY;
        b.out_tokens[to] = -1;
        b.out_parents[to] = 0;
        if (b.out_done) b.out_done[to] = 1;
    }
    if (!b.history) return;
    const int len = min(max(b.lengths[group], 0), b.history_len);
    for (int k = blockIdx.y; k < top; k += gridDim.y) {
        if (parent_of[k] < 0) continue;
        const int32_t* from = b.history + (size_t(group) * b.beams + parent_of[k]) * b.history_len;
        int32_t* to = b.out_history + (size_t(group) * top + k) * b.history_len;
        for (int i = tid; i < len; i += blockDim.x * kHistoryLoads) {
            int32_t v[kHistoryLoads];
#pragma unroll
            for (int u = 0; u < kHistoryLoads; ++u) v[u] = from[min(i + u * int(blockDim.x), len - 1)];
#pragma unroll
            for (int u = 0; u < kHistoryLoads; ++u)
                if (i + u * int(blockDim.x) < len) to[i + u * blockDim.x] = v[u];
        }
        if (tid == 0 && len < b.history_len) to[len] = token_of[k];
    }
}

}  // namespace card
