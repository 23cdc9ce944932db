// Attention of the new tokens of a ragged batch over one paged cache.
#pragma once
#include "card_common.hip"

namespace card {

struct AttendArgs {
    const void* q;
    const void* k;
    const void* v;
    void* out;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
    __bf16* kpool;  // of the layer
    __bf16* vpool;
    const int32_t* tables;
    const int32_t* ctx;
    const int32_t* starts;
    int32_t table_pages, n_pages, n_seqs, n_rows, G, Hkv;
    const uint32_t* mask;
    const int32_t* mask_base;
    int32_t mask_words;
    float scale;  // log2(e) / sqrt(head size): the softmax runs on exp2
};

// The sequence and the part of it that unit number `unit` of a launch is about.  Units are dealt so that no prefix sum is needed:
// sequence s has the units from floor(start_s * mul / div) + add * s on, which are enough for ceil(new_s * mul / div) + add - 1 of them.
struct SeqUnit {
    int32_t seq, index, row0, n_new, ctx, len;
};
__device__ __forceinline__ int32_t seq_start(const AttendArgs& a, int s) {
    return min(max(a.starts[s], 0), a.n_rows);
}
__device__ __forceinline__ SeqUnit find_unit(const AttendArgs& a, int unit, int mul, int div, int add) {
    const int lane = threadIdx.x & 63;
    const auto first = [&](int s) { return int(int64_t(seq_start(a, s)) * mul / div) + add * s; };
    int lo = 0, hi = a.n_seqs;  // 64 places are looked at at a time: one load up to 64 sequences
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) >> 6, s = lo + lane * step;
        const int hits = __popcll(__ballot(s < hi && first(s) <= unit));
        lo += max(hits - 1, 0) * step;
        hi = min(hi, lo + step);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    SeqUnit u;
    u.seq = lo;
    u.index = unit - first(lo);
    u.row0 = seq_start(a, lo);
    u.n_new = max(seq_start(a, lo + 1) - u.row0, 0);
    const int room = a.table_pages * 16;
    u.ctx = min(max(a.ctx[lo], 0), room);
    u.len = min(u.ctx + u.n_new, room);
    return u;
}

// Keys and values of the new tokens go to their pages.  One workgroup: one page of one KV head.  A thread writes the 8 elements of a token
// that lie together in K, or the 4 tokens of an element that lie together in V.
constexpr int kStoreUnits = 2;  // pages per sequence beyond its new tokens / 16
template <typename T>
__global__ __launch_bounds__(256) void k_attend_store(AttendArgs a, int h) {
    const SeqUnit u = find_unit(a, blockIdx.x, 1, 16, kStoreUnits);
    if (u.index < 0 || u.len <= u.ctx) return;
    const int pg = (u.ctx >> 4) + u.index, slot0 = pg * 16, head = blockIdx.y;
    if (slot0 >= u.len) return;
    const int page = a.tables[int64_t(u.seq) * a.table_pages + pg];
    if (page < 0 || page >= a.n_pages) return;
    const int t0 = max(u.ctx - slot0, 0), t1 = min(u.len - slot0, 16);  // the places of new tokens
    const int64_t row0 = int64_t(u.row0) + slot0 - u.ctx;  // the row of place 0
    const size_t base = (size_t(page) * a.Hkv + head) * (16 * h);
    const T* k = static_cast<const T*>(a.k) + head * a.k_head;
    const T* v = static_cast<const T*>(a.v) + head * a.v_head;
    for (int e = threadIdx.x; e < 2 * h; e += 256) {
        const int t = e & 15, jg = e >> 4;
        if (t < t0 || t >= t1) continue;
        const T* p = k + (row0 + t) * a.k_row + jg * 8;
        bf16x8 w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = static_cast<__bf16>(p[i]);
        *reinterpret_cast<bf16x8*>(a.kpool + base + e * 8) = w;
    }
    for (int e = threadIdx.x; e < 4 * h; e += 256) {
        const int j = e % h, t = e / h * 4;
        __bf16* to = a.vpool + base + v_page_index(j, t);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i >= t0 && t + i < t1) to[i] = static_cast<__bf16>(v[(row0 + t + i) * a.v_row + j]);
    }
}

// A float as the sum of N bf16: of one part 8 bits of it, of three all 24.
template <int N>
__device__ __forceinline__ void split_parts(float v, __bf16 (&p)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        p[i] = static_cast<__bf16>(v);
        v -= static_cast<float>(p[i]);
    }
}

// Which of the four keys from slot on a row sees.  limit: its own slot (causal), or the last one of the sequence.
__device__ __forceinline__ void seen_keys(const AttendArgs& a, int row, int base, int limit, int slot, bool (&ok)[4]) {
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        bool on = slot + v <= limit;
        if (a.mask) {
            const int bit = slot + v - base;
            if (on && bit >= 0) on = bit < 32 * a.mask_words && (a.mask[int64_t(row) * a.mask_words + (bit >> 5)] >> (bit & 31) & 1u);
        }
        ok[v] = on;
    }
}

// One wavefront: 16 rows x heads that share a KV head (number m * G + g: head g of new token m), all pages that the last of them sees.
template <int H, typename T>
__global__ __launch_bounds__(64) void k_attend(AttendArgs a) {
    constexpr int ST = H / 32, HT = H / 16, NP = sizeof(T) == 4 ? 3 : 1;
    const int lane = threadIdx.x, col = lane & 15, kq = lane >> 4, kvh = blockIdx.y;
    const SeqUnit u = find_unit(a, blockIdx.x, a.G, 16, 1);
    const int R = u.n_new * a.G, rho = u.index * 16 + col;
    if (u.index < 0 || u.index * 16 >= R) return;
    const bool row_ok = rho < R;
    const int m = row_ok ? rho / a.G : 0, head = kvh * a.G + (row_ok ? rho % a.G : 0), row = u.row0 + m;
    const int base = a.mask ? max(a.mask_base[u.seq], 0) : 0;
    const int limit = row_ok ? (a.mask ? u.len - 1 : min(u.ctx + m, u.len - 1)) : -1;
    const int last = a.mask ? u.len - 1 : min(u.ctx + min(u.index * 16 + 15, R - 1) / a.G, u.len - 1);
    bf16x8 qf[NP][ST];
    {
        const T* p = static_cast<const T*>(a.q) + int64_t(row) * a.q_row + int64_t(head) * a.q_head + kq * 8;
#pragma unroll
        for (int st = 0; st < ST; ++st)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                __bf16 w[NP];
                split_parts<NP>(static_cast<float>(p[st * 32 + e]), w);
#pragma unroll
                for (int i = 0; i < NP; ++i) qf[i][st][e] = w[i];
            }
    }
    floatx4 o[HT];
#pragma unroll
    for (int i = 0; i < HT; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    float mx = -INFINITY, sum = 0.f;
    for (int pg = 0; pg * 16 <= last; ++pg) {
        const int id = a.tables[int64_t(u.seq) * a.table_pages + pg];
        const bool held = id >= 0 && id < a.n_pages;
        const size_t at = (size_t(held ? id : 0) * a.Hkv + kvh) * (16 * H);
        const bf16x8* kp = reinterpret_cast<const bf16x8*>(a.kpool + at) + lane;
        const short4v* vp = reinterpret_cast<const short4v*>(a.vpool + at) + lane * 2;
        floatx4 s = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < ST; ++st)
#pragma unroll
            for (int i = 0; i < NP; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kp[st * 64], qf[i][st], s, 0, 0, 0);
        bool ok[4];
        seen_keys(a, row, base, held ? limit : -1, pg * 16 + kq * 4, ok);
        float pmax = -INFINITY;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            s[v] *= a.scale;
            if (ok[v]) pmax = fmaxf(pmax, s[v]);
        }
        const float mnew = fmaxf(mx, max_across_rows(pmax)), mref = mnew == -INFINITY ? 0.f : mnew;
        const float alpha = __builtin_amdgcn_exp2f(mx - mref);
        float psum = 0.f;
        short4v p[NP];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const float x = ok[v] ? __builtin_amdgcn_exp2f(s[v] - mref) : 0.f;
            psum += x;
            __bf16 w[NP];
            split_parts<NP>(x, w);
#pragma unroll
            for (int i = 0; i < NP; ++i) p[i][v] = __builtin_bit_cast(short, w[i]);
        }
        sum = sum * alpha + sum_across_rows(psum);
        mx = mnew;
        // (slots behind the sequence's end may hold anything: not multiplied, not even by zero)
        const int there = held ? u.len - pg * 16 - kq * 4 : 0;
#pragma unroll
        for (int i = 0; i < HT; ++i) {
            short4v w = vp[(i >> 1) * 128 + (i & 1)];
#pragma unroll
            for (int v = 0; v < 4; ++v) w[v] = v < there ? w[v] : short(0);
            floatx4 acc = o[i] * alpha;
#pragma unroll
            for (int n = 0; n < NP; ++n) acc = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(w, p[n], acc, 0, 0, 0);
            o[i] = acc;
        }
    }
    if (!row_ok) return;
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    T* to = static_cast<T*>(a.out) + int64_t(row) * a.o_row + int64_t(head) * a.o_head + kq * 4;
#pragma unroll
    for (int i = 0; i < HT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[i * 16 + e] = static_cast<T>(o[i][e] * inv);
}

}  // namespace card
