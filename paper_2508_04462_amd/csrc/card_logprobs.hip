// Log probabilities, entropies and most probable tokens of rows of logits.
#pragma once
#include "card_common.hip"

namespace card {

constexpr int kMaxTop = 32;

struct LogprobArgs {
    const void* logits;
    int64_t row_stride;
    int32_t vocab, top;
    const int32_t* tokens;
    float inv_temp;
    float* logprob;
    float* entropy;
    int32_t* top_tokens;
    float* top_logprobs;
};

__device__ __forceinline__ float logit_at(const float* p, int i) { return p[i]; }
__device__ __forceinline__ float logit_at(const __bf16* p, int i) { return static_cast<float>(p[i]); }

// (max, sum of e^d, sum of d e^d) of one part of a row, d = (x - max) / T; a NaN anywhere is in the sum.
struct RowSums {
    float m, s, t;
};
// d is kept finite where it meets e^d = 0: a logit of -inf (or far below) has no part in either sum
__device__ __forceinline__ RowSums join_sums(RowSums a, RowSums b, float inv_temp) {
    const float m = fmaxf(a.m, b.m);
    const float da = fmaxf((a.m - m) * inv_temp, -1e4f), db = fmaxf((b.m - m) * inv_temp, -1e4f);
    const float ea = expf((a.m - m) * inv_temp), eb = expf((b.m - m) * inv_temp);
    return {m, a.s * ea + b.s * eb, (a.t + a.s * da) * ea + (b.t + b.s * db) * eb};
}

// One workgroup: one row; a pass for the sums, then one for each of the most probable tokens.
template <typename T>
__global__ __launch_bounds__(256) void k_logprobs(LogprobArgs a) {
    __shared__ RowSums sums[256];
    __shared__ unsigned long long best[256];
    const int row = blockIdx.x, tid = threadIdx.x;
    const T* x = static_cast<const T*>(a.logits) + int64_t(row) * a.row_stride;
    RowSums r = {-3.402823466e38f, 0.f, 0.f};
    for (int i = tid; i < a.vocab; i += 256) r = join_sums(r, RowSums{logit_at(x, i) == -INFINITY ? -3.402823466e38f : logit_at(x, i), logit_at(x, i) == -INFINITY ? 0.f : 1.f, 0.f}, a.inv_temp);
    sums[tid] = r;
    __syncthreads();
    for (int d = 128; d > 0; d >>= 1) {
        if (tid < d) sums[tid] = join_sums(sums[tid], sums[tid + d], a.inv_temp);
        __syncthreads();
    }
    r = sums[0];
    const float ln_s = logf(r.s);
    const bool is_void = r.s != r.s || r.m == INFINITY, empty = r.s == 0.f;
    const auto logprob = [&](float v) { return is_void ? NAN : (empty ? -INFINITY : (v - r.m) * a.inv_temp - ln_s); };
    if (tid == 0) {
        if (a.tokens) {
            const int tok = a.tokens[row];
            a.logprob[row] = tok < 0 ? 0.f : (tok >= a.vocab ? NAN : logprob(logit_at(x, tok)));
        }
        if (a.entropy) a.entropy[row] = is_void ? NAN : (empty ? 0.f : ln_s - r.t / r.s);
    }
    unsigned long long below = ~0ull;
    for (int k = 0; k < a.top; ++k) {
        unsigned long long b = 0ull;
        for (int i = tid; i < a.vocab; i += 256) {
            const float v = logit_at(x, i);
            const unsigned long long key = (static_cast<unsigned long long>(float_key(v + 0.f)) << 32) | (0xffffffffu - uint32_t(i));
            if (v > -INFINITY && key < below && key > b) b = key;
        }
        best[tid] = b;
        __syncthreads();
        for (int d = 128; d > 0; d >>= 1) {
            if (tid < d && best[tid + d] > best[tid]) best[tid] = best[tid + d];
            __syncthreads();
        }
        b = best[0];
        __syncthreads();
        if (tid == 0) {
            const int tok = int(0xffffffffu - uint32_t(b));
            const bool none = b == 0ull || is_void;
            a.top_tokens[int64_t(row) * a.top + k] = none ? -1 : tok;
            a.top_logprobs[int64_t(row) * a.top + k] = is_void ? NAN : (none ? -INFINITY : logprob(logit_at(x, tok)));
        }
        below = b;
    }
}

}  // namespace card
