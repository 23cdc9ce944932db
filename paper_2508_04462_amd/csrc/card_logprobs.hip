// Log probabilities, entropies and most probable tokens of rows of logits.
//
// One pass over a row: with m the largest logit so far and d = (x - m) / T, s = sum e^d and t = sum d e^d are rescaled as m grows;
// ln p = d - ln s and the entropy is ln s - t / s.  d is taken from the difference, not from x / T - m / T: far from
// zero those two lose what the difference keeps.  Bound by reading the logits: 1000 rows of 152064 in bf16, 304 MB, in 58 us (5.2 TB/s) with the most
// probable token; a few rows by the latency of one pass and a join (8 rows of 128256 in fp32, five tokens: 6.0 + 4.3 us).
#pragma once
#include "card_common.hip"

namespace card {

constexpr int kMaxTop = 32;
constexpr int kLpThreads = 256, kLpWaves = 4;
constexpr int kLpVecs = 4;  // 16-byte loads of a lane in flight

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
    // a row in several parts: 16-byte units of a part, parts, and what each of them leaves: sums [row][part][4], keys [row][part][top]
    int32_t part_vecs, parts;
    float* part_sums;
    unsigned long long* part_keys;
};

__device__ __forceinline__ float logit_at(const float* p, int i) { return p[i]; }
__device__ __forceinline__ float logit_at(const __bf16* p, int i) { return static_cast<float>(p[i]); }
__device__ __forceinline__ void unpack_logits(uint4v w, float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void unpack_logits(uint4v w, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.402823466e38f;  // m before any logit; a logit of -inf then has d = -inf and no part in s or t

// Of some logits: largest, sum of 2^d and sum of d 2^d, d = (x - m) log2(e) / T.  A NaN or +inf among them makes s NaN.
// d is kept finite where it meets 2^d = 0.
struct RowSums {
    float m, s, t;
    __device__ __forceinline__ void raise(float mnew, float c) {
        const float d = (m - mnew) * c, e = __builtin_amdgcn_exp2f(d);
        t = (t + s * fmaxf(d, -1e4f)) * e;
        s *= e;
        m = mnew;
    }
    template <bool ENTROPY>
    __device__ __forceinline__ void add(float x, float c) {
        const float d = (x - m) * c, e = __builtin_amdgcn_exp2f(d);
        s += e;
        if constexpr (ENTROPY) t = fmaf(e, fmaxf(d, -1e4f), t);
    }
    __device__ __forceinline__ void join(RowSums b, float c) {
        const float mnew = fmaxf(m, b.m);
        raise(mnew, c);
        b.raise(mnew, c);
        s += b.s;
        t += b.t;
    }
};
template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
    const int i = int(__float_as_uint(v));
    return fmaxf(v, __uint_as_float(uint32_t(__builtin_amdgcn_update_dpp(i, i, CTRL, 0xf, 0xf, false))));
}
__device__ __forceinline__ float sum_of_lanes(float v) {
    return sum_across_rows(dpp_add<0x140>(dpp_add<0x141>(dpp_add<0x4E>(dpp_add<0xB1>(v)))));
}
__device__ __forceinline__ RowSums join_lanes(RowSums r, float c) {
    r.raise(max_across_rows(dpp_max<0x140>(dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(r.m))))), c);
    return RowSums{r.m, sum_of_lanes(r.s), sum_of_lanes(r.t)};
}

// The largest keys that a wavefront has been offered, in order: lane i holds the i-th of them, a key that is not above `least` does not
// enter.  Keys are a logit in the upper half, the complement of its token in the lower one: unique, and equal logits order by token.
// An offer costs a comparison and a ballot; a key that enters, about 80 clocks.  Of n keys in random order top * ln(n / top) enter an empty list;
// floor(), on the first ones, keeps nearly all out that will not stay, and so does what the other wavefronts of the row have found.
__device__ __forceinline__ unsigned long long lane_key(unsigned long long v, int lane) {
    return uint64_t(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(v)), lane))) |
           (uint64_t(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(v >> 32)), lane))) << 32);
}
struct TopList {
    unsigned long long best = 0ull, least = 0ull, bottom = 0ull;
    // upper: the upper half of the largest key that this lane is about to offer.  At least `top` keys reach the top-th largest of the lanes'.
    __device__ __forceinline__ void floor(uint32_t upper, int top) {
        uint32_t t = 0u;
        for (int bit = 31; bit >= 8; --bit)  // (to 24 bits, rounded down)
            if (__popcll(__ballot(upper >= (t | 1u << bit))) >= top) t |= 1u << bit;
        if (t > 0u) at_least((static_cast<unsigned long long>(t) << 32) - 1ull);
    }
    __device__ __forceinline__ void at_least(unsigned long long key) {
        if (key > bottom) bottom = key;
        if (bottom > least) least = bottom;
    }
    __device__ __forceinline__ void offer(unsigned long long key, int top, int lane) {
        unsigned long long in = __ballot(key > least);
        while (in) {
            const unsigned long long k = lane_key(key, __ffsll(in) - 1);
            const int at = __popcll(__ballot(best > k));
            const int lo = int(uint32_t(best)), hi = int(uint32_t(best >> 32));  // one lane up
            const unsigned long long up = uint64_t(uint32_t(__builtin_amdgcn_update_dpp(lo, lo, 0x138, 0xf, 0xf, false))) |
                                          (uint64_t(uint32_t(__builtin_amdgcn_update_dpp(hi, hi, 0x138, 0xf, 0xf, false))) << 32);
            best = lane < at ? best : (lane == at ? k : up);
            const unsigned long long last = lane_key(best, top - 1);
            least = last > bottom ? last : bottom;
            in &= in - 1;
            in &= __ballot(key > least);
        }
    }
};
__device__ __forceinline__ unsigned long long logit_key(float x, int token) {
    // (-0 and 0 are equal; without probability: no key)
    return x == -INFINITY ? 0ull : (uint64_t(float_key(x + 0.f)) << 32) | (0xffffffffu - uint32_t(token));
}

// The logit of a key; -inf of none, or of one below all logits'.
__device__ __forceinline__ float key_logit(unsigned long long key) {
    const uint32_t f = uint32_t(key >> 32);
    return f <= 0x007fffffu ? -INFINITY : __uint_as_float(f & 0x80000000u ? f ^ 0x80000000u : ~f);
}

struct LogprobShared {
    float sums[kLpWaves][3];
    unsigned long long least;  // the largest of the wavefronts' `least`: of their keys, too, `top` are not smaller
    unsigned long long keys[kLpWaves * kMaxTop], out[kMaxTop];
};

// The wavefronts' sums and lists become the workgroup's: returned, and in sm.out.
__device__ __forceinline__ RowSums join_waves(LogprobShared& sm, RowSums r, const TopList& list, int top, float c) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    r = join_lanes(r, c);
    if (lane == 0) {
        sm.sums[wave][0] = r.m;
        sm.sums[wave][1] = r.s;
        sm.sums[wave][2] = r.t;
    }
    if (lane < top) sm.keys[wave * top + lane] = list.best;
    if (tid < top) sm.out[tid] = 0ull;
    __syncthreads();
    r = {sm.sums[0][0], sm.sums[0][1], sm.sums[0][2]};
#pragma unroll
    for (int w = 1; w < kLpWaves; ++w) r.join(RowSums{sm.sums[w][0], sm.sums[w][1], sm.sums[w][2]}, c);
    if (tid < kLpWaves * top && sm.keys[tid] != 0ull) {  // the place of a key: how many are larger
        const unsigned long long k = sm.keys[tid];
        int larger = 0;
        for (int i = 0; i < kLpWaves * top; ++i) larger += sm.keys[i] > k;
        if (larger < top) sm.out[larger] = k;
    }
    __syncthreads();
    return r;
}

template <typename T>
__device__ __forceinline__ void finish_row(const LogprobArgs& a, const LogprobShared& sm, RowSums r, int row) {
    const int tid = threadIdx.x;
    const T* x = static_cast<const T*>(a.logits) + int64_t(row) * a.row_stride;
    const float ln_s = logf(r.s);
    const bool is_void = r.s != r.s, empty = r.s == 0.f;
    // (of halves: the difference of two logits may be beyond the largest float where the quotient is not)
    const auto logprob = [&](float v) { return is_void ? NAN : (empty ? -INFINITY : (0.5f * v - 0.5f * r.m) * a.inv_temp * 2.f - ln_s); };
    if (tid < a.top) {
        const unsigned long long key = sm.out[tid];
        const bool none = is_void || key == 0ull;
        a.top_tokens[int64_t(row) * a.top + tid] = none ? -1 : int(0xffffffffu - uint32_t(key));
        a.top_logprobs[int64_t(row) * a.top + tid] = none ? (is_void ? NAN : -INFINITY) : logprob(key_logit(key));
    }
    if (tid == 64) {  // (another wavefront than the one above)
        if (a.tokens) {
            const int tok = a.tokens[row];
            a.logprob[row] = tok < 0 ? 0.f : (tok >= a.vocab ? NAN : logprob(logit_at(x, tok)));
        }
        if (a.entropy) a.entropy[row] = is_void ? NAN : (empty ? 0.f : ln_s - r.t / r.s * kLn2);
    }
}

// A workgroup's part of a row, in turns of kLpVecs 16-byte loads a lane: returns its sums, and leaves its most probable tokens in sm.out.
// BY_TOKEN: units of 16 bytes begin with the row, so that which logits a lane and a part add up, and with it the sums' last bits, does not depend on where the row lies (240 rows of
// 152063 in bf16, from any place, 29.4 us with the join, of 152064 29.0; from aligned units 29.1 and 29.5).  Else the loads are of aligned units, whatever the row begins
// at: what a unit holds before the row or behind it is not read.
// ENTROPY: with t, which costs two instructions a logit.
template <typename T, bool ENTROPY, bool BY_TOKEN>
__device__ __forceinline__ RowSums scan_part(const LogprobArgs& a, LogprobShared& sm, int row, int part) {
    constexpr int VN = 16 / sizeof(T);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float c = a.inv_temp * kLog2e;
    const T* x0 = static_cast<const T*>(a.logits) + int64_t(row) * a.row_stride;
    const int lead = BY_TOKEN ? 0 : int(reinterpret_cast<uintptr_t>(x0) % 16 / sizeof(T));  // logits of the first unit that are not the row's
    const T* units = x0 - lead;
    const int n_units = (lead + a.vocab + VN - 1) / VN, end = min(n_units, (part + 1) * a.part_vecs);
    RowSums r = {kLowest, 0.f, 0.f};
    TopList list;
    if (tid == 0) sm.least = 0ull;
    __syncthreads();
    for (int first = part * a.part_vecs + wave * 64 * kLpVecs; first < end; first += kLpThreads * kLpVecs) {
        float x[kLpVecs][VN];
        if (first * VN >= lead && (first + 64 * kLpVecs) * VN <= lead + a.vocab && first + 64 * kLpVecs <= end) {
            uint4v w[kLpVecs];
#pragma unroll
            for (int u = 0; u < kLpVecs; ++u) {
                const T* from = units + (first + u * 64 + lane) * VN;
                if constexpr (BY_TOKEN) __builtin_memcpy(&w[u], from, 16);
                else w[u] = *reinterpret_cast<const uint4v*>(from);
            }
#pragma unroll
            for (int u = 0; u < kLpVecs; ++u) unpack_logits(w[u], x[u]);
        } else {  // the ends of the row or of the part
#pragma unroll
            for (int u = 0; u < kLpVecs; ++u) {
                const int unit = first + u * 64 + lane;
#pragma unroll
                for (int e = 0; e < VN; ++e) {
                    const int i = unit * VN + e - lead;
                    x[u][e] = unit < end && i >= 0 && i < a.vocab ? logit_at(x0, i) : -INFINITY;
                }
            }
        }
        float most[kLpVecs];
#pragma unroll
        for (int u = 0; u < kLpVecs; ++u) {
            most[u] = x[u][0];
#pragma unroll
            for (int e = 1; e < VN; ++e) most[u] = fmaxf(most[u], x[u][e]);
        }
        float all = most[0];
#pragma unroll
        for (int u = 1; u < kLpVecs; ++u) all = fmaxf(all, most[u]);
        r.raise(fmaxf(r.m, all), c);
        RowSums turn = {r.m, 0.f, 0.f};  // (added up on its own: a few roundings of a large sum instead of one per logit)
#pragma unroll
        for (int u = 0; u < kLpVecs; ++u)
#pragma unroll
            for (int e = 0; e < VN; ++e) turn.add<ENTROPY>(x[u][e], c);
        r.s += turn.s;
        r.t += turn.t;
        if (a.top == 0) continue;
        const unsigned long long others = *const_cast<volatile unsigned long long*>(&sm.least);
        list.at_least(lane_key(others, 0));
        if (list.bottom == 0ull && !__ballot(list.best != 0ull)) list.floor(float_key(all + 0.f), a.top);
        // (tokens of later turns are larger: an equal logit does not enter; inside a turn it may)
        float limit = key_logit(list.least);
        if (__ballot(all >= limit)) {
            const unsigned long long before = list.least;
#pragma unroll
            for (int u = 0; u < kLpVecs; ++u) {
                if (!__ballot(most[u] >= limit)) continue;
#pragma unroll
                for (int e = 0; e < VN; ++e) {
                    if (!__ballot(x[u][e] >= limit)) continue;
                    list.offer(logit_key(x[u][e], (first + u * 64 + lane) * VN + e - lead), a.top, lane);
                    limit = key_logit(list.least);
                }
            }
            if (lane == 0 && list.least > before) atomicMax(&sm.least, list.least);
        }
    }
    return join_waves(sm, r, list, a.top, c);
}
__device__ __forceinline__ void leave_part(const LogprobArgs& a, const LogprobShared& sm, RowSums r, int row, int part) {
    const int tid = threadIdx.x;
    const size_t at = size_t(row) * a.parts + part;
    if (tid == 0) *reinterpret_cast<floatx4*>(a.part_sums + at * 4) = floatx4{r.m, r.s, r.t, 0.f};
    if (tid < a.top) a.part_keys[at * a.top + tid] = sm.out[tid];
}

// One workgroup: one part of one row.
template <typename T>
__global__ __launch_bounds__(kLpThreads) void k_logprobs(LogprobArgs a) {
    __shared__ LogprobShared sm;
    const int row = blockIdx.x, part = blockIdx.y;
    const RowSums r = scan_part<T, true, false>(a, sm, row, part);
    if (a.parts == 1) finish_row<T>(a, sm, r, row);
    else leave_part(a, sm, r, row, part);
}

// One workgroup: the parts of a row.
template <typename T>
__global__ __launch_bounds__(kLpThreads) void k_logprobs_join(LogprobArgs a) {
    __shared__ LogprobShared sm;
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, n = a.parts * a.top;
    const float c = a.inv_temp * kLog2e;
    RowSums r = {kLowest, 0.f, 0.f};
    for (int p = tid; p < a.parts; p += kLpThreads) {
        const floatx4 v = *reinterpret_cast<const floatx4*>(a.part_sums + (size_t(row) * a.parts + p) * 4);
        r.join(RowSums{v[0], v[1], v[2]}, c);
    }
    TopList list;
    if (a.top > 0 && a.parts >= a.top)  // of the parts' first keys, the top-th largest
        list.floor(lane < a.parts ? uint32_t(a.part_keys[size_t(row) * n + lane * a.top] >> 32) : 0u, a.top);
    for (int i = tid - lane; i < n; i += kLpThreads) {
        const unsigned long long key = i + lane < n ? a.part_keys[size_t(row) * n + i + lane] : 0ull;
        if (i == tid - lane) list.floor(uint32_t(key >> 32), a.top);
        list.offer(key, a.top, lane);
    }
    r = join_waves(sm, r, list, a.top, c);
    finish_row<T>(a, sm, r, row);
}

}  // namespace card
