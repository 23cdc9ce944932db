// Attention of the new tokens of a ragged batch over one paged cache.
#pragma once
#include <type_traits>

#include "card_common.hip"

namespace card {

typedef __attribute__((ext_vector_type(2))) unsigned int uint2v;
typedef __attribute__((address_space(4))) int32_t const_i32;  // memory that no kernel writes meanwhile: scalar loads

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
    // the pages of a sequence in up to `cuts` cuts of cut_pages or more, and their partial results where there are several
    int32_t cuts, cut_pages;
    float* part;
};

__device__ __forceinline__ uint32_t bf16_bits(__bf16 v) { return __builtin_bit_cast(unsigned short, v); }

// The sequence and the part of it that unit number `unit` of a launch is about.  Units are dealt so that no prefix sum is needed:
// sequence s has the units from floor(start_s * mul / div) + add * s on, which are enough for ceil(new_s * mul / div) + add - 1 of them.
struct SeqUnit {
    int32_t seq, index, row0, n_new, ctx, len;
    int32_t held;  // tokens in the cache as the lengths say it; ctx: as far as the table goes
};
__device__ __forceinline__ int32_t seq_start(const AttendArgs& a, int s) {
    return min(max(a.starts[s], 0), a.n_rows);
}
__device__ __forceinline__ SeqUnit find_unit(const AttendArgs& a, int unit, int mul, int div, int add) {
    const int lane = threadIdx.x & 63;
    const auto first = [&](int start, int s) { return int(int64_t(start) * mul / div) + add * s; };
    int lo = 0, hi = a.n_seqs;
    while (hi - lo > 64) {  // 64 places are looked at at a time
        const int step = (hi - lo + 63) >> 6, s = lo + lane * step;
        const int hits = __popcll(__ballot(s < hi && first(seq_start(a, min(s, hi - 1)), s) <= unit));
        lo += max(hits - 1, 0) * step;
        hi = min(hi, lo + step);
    }
    // the last 64: all that is to be known of each, in one round trip
    const int s = min(lo + lane, hi - 1), start = seq_start(a, s), end = seq_start(a, s + 1), held = a.ctx[s];
    const int hits = __popcll(__ballot(lo + lane < hi && first(start, s) <= unit));  // (none: row starts that do not begin at 0)
    const int at = max(hits - 1, 0);
    SeqUnit u;
    u.seq = __builtin_amdgcn_readfirstlane(lo + at);
    u.row0 = __builtin_amdgcn_readlane(start, at);
    u.index = unit - first(u.row0, u.seq);
    u.n_new = max(__builtin_amdgcn_readlane(end, at) - u.row0, 0);
    const int room = a.table_pages * 16;
    u.held = max(__builtin_amdgcn_readlane(held, at), 0);
    u.ctx = min(u.held, room);
    u.len = min(u.ctx + u.n_new, room);
    return u;
}

// Keys and values of the new tokens go to their pages.  One workgroup: one page of one KV head.  A thread writes the 8 elements of a token
// that lie together in K, and the 4 tokens of an element that lie together in V; it reads all of them before it writes any: one
// round trip to memory, which bounds it (about 2280 bf16 rows of 4 heads of 128 in 7.1 us, against 8.0 with K written before V is read; 2000 rows of 8
// heads 7.1 against 7.6).
constexpr int kStoreUnits = 2;  // pages per sequence beyond its new tokens / 16
template <int H, typename T>
__global__ __launch_bounds__(256) void k_attend_store(AttendArgs a) {
    constexpr int KU = (2 * H + 255) / 256, VU = 4 * H / 256;  // of a thread, in K and in V
    const SeqUnit u = find_unit(a, blockIdx.x, 1, 16, kStoreUnits);
    if (u.index < 0 || u.len <= u.ctx) return;
    const int pg = (u.ctx >> 4) + u.index, slot0 = pg * 16, head = blockIdx.y;
    if (slot0 >= u.len) return;
    const int page = a.tables[int64_t(u.seq) * a.table_pages + pg];
    const int t0 = max(u.ctx - slot0, 0), t1 = min(u.len - slot0, 16);  // the places of new tokens
    const int64_t row0 = int64_t(u.row0) + slot0 - u.ctx;  // the row of place 0
    const T* k = static_cast<const T*>(a.k) + head * a.k_head;
    const T* v = static_cast<const T*>(a.v) + head * a.v_head;
    bf16x8 wk[KU];
    __bf16 wv[VU][4];
#pragma unroll
    for (int x = 0; x < KU; ++x) {
        const int e = min(x * 256 + int(threadIdx.x), 2 * H - 1);
        const T* p = k + (row0 + min(max(e & 15, t0), t1 - 1)) * a.k_row + (e >> 4) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) wk[x][i] = static_cast<__bf16>(p[i]);
    }
#pragma unroll
    for (int x = 0; x < VU; ++x) {
        const int e = x * 256 + threadIdx.x, j = e % H, t = e / H * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) wv[x][i] = static_cast<__bf16>(v[(row0 + min(max(t + i, t0), t1 - 1)) * a.v_row + j]);
    }
    if (page < 0 || page >= a.n_pages) return;
    const size_t base = (size_t(page) * a.Hkv + head) * (16 * H);
#pragma unroll
    for (int x = 0; x < KU; ++x) {
        const int e = x * 256 + threadIdx.x, t = e & 15;
        if (e < 2 * H && t >= t0 && t < t1) *reinterpret_cast<bf16x8*>(a.kpool + base + e * 8) = wk[x];
    }
#pragma unroll
    for (int x = 0; x < VU; ++x) {
        const int e = x * 256 + threadIdx.x, j = e % H, t = e / H * 4;
        __bf16* to = a.vpool + base + v_page_index(j, t);
        const __bf16* w = wv[x];
        if (t >= t0 && t + 4 <= t1) {
            *reinterpret_cast<uint2v*>(to) = uint2v{bf16_bits(w[0]) | bf16_bits(w[1]) << 16, bf16_bits(w[2]) | bf16_bits(w[3]) << 16};
            continue;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i >= t0 && t + i < t1) to[i] = w[i];
    }
}

// Two floats as sums of N bf16, a pair in each word: of one part 8 bits of them, of two 16, of three all 24.
template <int N>
__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t (&p)[N]) {
    typedef __attribute__((ext_vector_type(2))) float float2v;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        p[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{x0, x1}), bf16x2));
        if (i + 1 < N) {
            x0 -= __uint_as_float(p[i] << 16);
            x1 -= __uint_as_float(p[i] & 0xffff0000u);
        }
    }
}
__device__ __forceinline__ uint32_t pack_pair(float x0, float x1) {
    uint32_t p[1];
    split_pair<1>(x0, x1, p);
    return p[0];
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

// The rows x heads that share a KV head (number m * G + g: head g of new token m) in tiles of 16: lane l of a wavefront belongs to column
// l % 16 of each, and holds of the scores S^T = K Q^T of a page four keys, 4 (l / 16) .. + 3, as P V takes them.
struct Column {
    bool ok;
    int32_t row, head, limit;  // its row of the call; the last slot that it sees without a mask
};
__device__ __forceinline__ Column column_of(const AttendArgs& a, const SeqUnit& u, int kvh, int rho) {
    Column c;
    c.ok = rho < u.n_new * a.G;
    const int m = c.ok ? rho / a.G : 0;
    c.row = u.row0 + m;
    c.head = kvh * a.G + (c.ok ? rho % a.G : 0);
    c.limit = a.mask ? u.len - 1 : min(u.ctx + m, u.len - 1);
    return c;
}
template <int H, typename T, int NP>
__device__ __forceinline__ void load_query(const AttendArgs& a, const Column& c, int kq, bf16x8 (&qf)[NP][H / 32]) {
    const T* p = static_cast<const T*>(a.q) + int64_t(c.row) * a.q_row + int64_t(c.head) * a.q_head + kq * 8;
#pragma unroll
    for (int st = 0; st < H / 32; ++st) {
        uint4v w[NP];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t pair[NP];
            split_pair<NP>(static_cast<float>(p[st * 32 + 2 * e]), static_cast<float>(p[st * 32 + 2 * e + 1]), pair);
#pragma unroll
            for (int i = 0; i < NP; ++i) w[i][e] = pair[i];
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) qf[i][st] = __builtin_bit_cast(bf16x8, w[i]);
    }
}
template <int H>
__device__ __forceinline__ void load_k_page(const AttendArgs& a, int id, int kvh, int lane, bf16x8 (&k)[H / 32]) {
    const bf16x8* p = reinterpret_cast<const bf16x8*>(a.kpool + (size_t(id) * a.Hkv + kvh) * (16 * H)) + lane;
#pragma unroll
    for (int st = 0; st < H / 32; ++st) k[st] = p[st * 64];
}
template <int H>
__device__ __forceinline__ void load_v_page(const AttendArgs& a, int id, int kvh, int lane, uint2v (&v)[H / 16]) {
    const uint4v* p = reinterpret_cast<const uint4v*>(a.vpool + (size_t(id) * a.Hkv + kvh) * (16 * H)) + lane;
#pragma unroll
    for (int i = 0; i < H / 32; ++i) {
        const uint4v w = p[i * 64];
        v[2 * i] = uint2v{w[0], w[1]};
        v[2 * i + 1] = uint2v{w[2], w[3]};
    }
}
// Of four values of 16 bits: those below number n, as a mask.
__device__ __forceinline__ uint2v first_of_four(int n) {
    return uint2v{(n > 0 ? 0xffffu : 0u) | (n > 1 ? 0xffff0000u : 0u), (n > 2 ? 0xffffu : 0u) | (n > 3 ? 0xffff0000u : 0u)};
}

// The new tokens of a workgroup's pages, from the call's arrays: in LDS for the rounds that need them, K as it lies, V transposed, by place in the
// cache so that the four tokens of a lane lie together; and in their pages, tokens [own0, own1), which are this workgroup's to store
// (whoever else reads the page takes them from the arrays, too).
constexpr int kStage = 64;
template <int H>
struct Stage {
    __bf16 k[kStage][H];
    __bf16 v[H][kStage + 4];
};
// Stores 8 elements of a token, from element c * 8 on.
template <int H>
__device__ __forceinline__ void store_token(const AttendArgs& a, const SeqUnit& u, int kvh, int slot, int c, bf16x8 k, bf16x8 v) {
    const int id = a.tables[int64_t(u.seq) * a.table_pages + (slot >> 4)];
    if (id < 0 || id >= a.n_pages) return;
    const size_t page = (size_t(id) * a.Hkv + kvh) * (16 * H);
    *reinterpret_cast<bf16x8*>(a.kpool + page + (c * 16 + (slot & 15)) * 8) = k;
#pragma unroll
    for (int i = 0; i < 8; ++i) a.vpool[page + v_page_index(c * 8 + i, slot & 15)] = v[i];
}
// What `use` does with 8 elements of each of the new tokens in slots [s0, s1): token, element / 8, key, value.
template <int H, typename T, typename F>
__device__ __forceinline__ void each_new_token(const AttendArgs& a, const SeqUnit& u, int kvh, int s0, int s1, F&& use) {
    const T* k = static_cast<const T*>(a.k) + int64_t(u.row0 - u.ctx) * a.k_row + int64_t(kvh) * a.k_head;
    const T* v = static_cast<const T*>(a.v) + int64_t(u.row0 - u.ctx) * a.v_row + int64_t(kvh) * a.v_head;
    for (int e = threadIdx.x; e < (s1 - s0) * (H / 8); e += 256) {
        const int slot = s0 + e / (H / 8), c = e % (H / 8);
        const T* pk = k + slot * a.k_row + c * 8;
        const T* pv = v + slot * a.v_row + c * 8;
        bf16x8 wk, wv;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            wk[i] = static_cast<__bf16>(pk[i]);
            wv[i] = static_cast<__bf16>(pv[i]);
        }
        use(slot, c, wk, wv);
    }
}
template <int H>
__device__ __forceinline__ void take_new_tokens(const SeqUnit& u, int slot, int lane, const Stage<H>& sm, bf16x8 (&k)[H / 32], uint2v (&v)[H / 16]) {
    const int col = lane & 15, kq = lane >> 4, tok = slot + col, t0 = slot + kq * 4;
    const bool fresh = tok >= u.ctx && tok < u.len;
    const int row = fresh ? tok - u.ctx : 0;
#pragma unroll
    for (int st = 0; st < H / 32; ++st) {
        const bf16x8 w = *reinterpret_cast<const bf16x8*>(&sm.k[row][st * 32 + kq * 8]);
        k[st] = fresh ? w : k[st];
    }
    const uint2v below = first_of_four(u.len - t0), old = first_of_four(u.ctx - t0), take = {below[0] & ~old[0], below[1] & ~old[1]};
    const int at = min(max(t0 - (u.ctx & ~3), 0), kStage);
#pragma unroll
    for (int i = 0; i < H / 16; ++i) {
        const uint2v w = *reinterpret_cast<const uint2v*>(&sm.v[i * 16 + col][at]);
        v[i] = (v[i] & ~take) | (w & take);
    }
}

// The pages that rows up to token m_last see, and their cuts.
struct UnitCuts {
    int32_t all_pages, pages, n;
};
__device__ __forceinline__ UnitCuts cuts_of(const AttendArgs& a, const SeqUnit& u, int m_last) {
    UnitCuts c;
    c.all_pages = ((a.mask ? u.len : min(u.ctx + m_last + 1, u.len)) + 15) >> 4;
    c.pages = max(a.cut_pages, (c.all_pages + a.cuts - 1) / a.cuts);
    c.n = (c.all_pages + c.pages - 1) / c.pages;
    return c;
}

// Scores, maxima, sums and output are held in fp32.  The weights go into P V as the sum of several bf16 parts (split_pair): with bf16 rows two, 16 bits, as
// the library's own steps and prompts take theirs, so that rounding the output to bf16 is what its error consists of (a batch against 64 bits, of the
// root mean square: 1.65e-3, an fp32 softmax rounded to bf16 1.65e-3; with one part 2.3e-3); with fp32 rows three, 24 bits, and q as well.  The
// sum of the weights takes them in 32 bits, or where it is a product with ones in the same parts, 2^-17 from that at most.  The second part
// costs nothing where the cache's reading binds (48 texts of a row each 94.2 us, with one part 94.1; 16 rows each 117, 115), and where the matrix
// units do what their third product takes (2000 rows x 4 behind 14000 tokens 649, 516).
template <typename T>
constexpr int kWeightParts = sizeof(T) == 4 ? 3 : 2;
constexpr float kSlack = 8.f;  // (see below; 0, k_attend_many: 649 -> 686 us, three texts of up to 1000 rows x 7 176 -> 199)

// Floats that a cut leaves of a tile: [16][H], [16] maxima, [16] sums.
template <int H>
constexpr int kPartFloats = 16 * (H + 2);

// For few rows per sequence (16 NT rows x heads of a KV head at a time): bound by reading the cache, so every page is read once, straight into
// the registers that the matrix instructions take it from.  One workgroup: one cut of the pages of a sequence, for one KV head; its four
// wavefronts take every fourth page each, two per round, and refill K as soon as the scores are done, V behind P V.  The wavefronts' results
// meet in LDS, the cuts' in memory, where k_attend_join adds them up.
// The KV heads of a unit are neighbours in the launch and so go to different compute dies: the dies' shares do not depend on how long which
// sequence is, and the workgroups of one head, which read the same pages, share an L2 (five rows x 8 behind 32700 tokens 37 us, with the units as neighbours
// 49; k_attend_many, 2000 rows x 4 behind 14000, weights in one part, 507 and 534; 48 texts of a row each 94.7 and 95.6).
// NEW: the call's keys and values are taken from its arrays and stored on the way; a kernel in front that stores them costs 2 us.
// 8 KV heads of 128: 48 texts of 400-4000 tokens, 444 MB, in 90 us (4.9 TB/s); 32700 tokens, 134 MB, in 28.
template <int H, typename T, int NT, bool NEW>
__global__ __launch_bounds__(256, NT * sizeof(T) == 2 ? 3 : 2) void k_attend_few(AttendArgs a) {
    constexpr int ST = H / 32, HT = H / 16, NP = sizeof(T) == 4 ? 3 : 1, NW = kWeightParts<T>, LD = H + 4, CH = H / 16;
    __shared__ union __align__(16) {
        Stage<H> stage;
        float red[4][16][LD];
    } sm;
    auto& red = sm.red;
    __shared__ float red_m[4][16], red_l[4][16];
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, kq = lane >> 4, cut = blockIdx.y;
    const int kvh = blockIdx.x % uint32_t(a.Hkv), at_unit = blockIdx.x / uint32_t(a.Hkv);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const SeqUnit u = find_unit(a, at_unit, a.G, 16 * NT, 1);
    const int R = u.n_new * a.G, rho0 = u.index * 16 * NT;
    if (u.index < 0 || rho0 >= R) return;
    const int m_first = rho0 / a.G, m_last = (min(rho0 + 16 * NT, R) - 1) / a.G;
    const UnitCuts uc = cuts_of(a, u, m_last);
    if (cut >= uc.n) return;
    const int p0 = cut * uc.pages + wave, p1 = min(uc.all_pages, (cut + 1) * uc.pages);
    const int base = a.mask ? max(a.mask_base[u.seq], 0) : 0;
    const int all_see = __builtin_amdgcn_readfirstlane(a.mask ? min(base, u.len) : min(u.ctx + m_first + 1, u.len));  // slots below are seen by every row
    const int own0 = u.ctx + (rho0 + a.G - 1) / a.G, own1 = u.ctx + m_last + 1;  // the tokens whose first head is among the rows
    bool fresh = NEW && p1 * 16 > u.ctx;  // new tokens among this cut's
    if (NEW && fresh && u.n_new > kStage) {  // more than max_new said: they go to their pages first (the same values by whoever reads them)
        each_new_token<H, T>(a, u, kvh, max(u.ctx, cut * uc.pages * 16), min(u.len, p1 * 16),
                             [&](int slot, int c, bf16x8 wk, bf16x8 wv) { store_token<H>(a, u, kvh, slot, c, wk, wv); });
        __threadfence_block();
        __syncthreads();
        fresh = false;
    }
    Column c[NT];
    bf16x8 qf[NT][NP][ST];
    floatx4 o[NT][HT];
    float mx[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        c[n] = column_of(a, u, kvh, rho0 + n * 16 + col);
        load_query<H, T, NP>(a, c[n], kq, qf[n]);
#pragma unroll
        for (int i = 0; i < HT; ++i) o[n][i] = floatx4{0.f, 0.f, 0.f, 0.f};
        mx[n] = -INFINITY;
        sum[n] = 0.f;
    }
    // page ids are scalar loads, a round ahead: they wait on a counter of their own, not on the pages under way
    const const_i32* table = reinterpret_cast<const const_i32*>(reinterpret_cast<uintptr_t>(a.tables + int64_t(u.seq) * a.table_pages));
    const int count = p0 < p1 ? (p1 - p0 + 3) >> 2 : 0;
    const auto page_id = [&](int i) { return i < count ? table[p0 + 4 * i] : -1; };
    const auto held = [&](int id) { return id >= 0 && id < a.n_pages; };
    // pages that hold no new token and that every row sees whole come first, in pairs: their rounds have no memory access but the
    // refills, which then stay in flight (the last round, which has none, goes with the others)
    const int plain_end = min(p1, min(fresh ? min(u.ctx, all_see) : all_see, u.len) >> 4);
    const int plain = min(p0 < plain_end ? (plain_end - p0 + 3) >> 2 : 0, count - 2) & ~1;
    bf16x8 k[2][ST];
    uint2v v[2][HT];
    int id[2], next_id[2];
    const auto refill_k = [&]() {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            id[j] = next_id[j];
            load_k_page<H>(a, held(id[j]) ? id[j] : 0, kvh, lane, k[j]);
        }
    };
    const auto refill_v = [&](int i) {  // of pages i and i + 1
#pragma unroll
        for (int j = 0; j < 2; ++j) load_v_page<H>(a, held(id[j]) ? id[j] : 0, kvh, lane, v[j]);
#pragma unroll
        for (int j = 0; j < 2; ++j) next_id[j] = page_id(i + 2 + j);
    };
    const auto round = [&](int i, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        int slot[2];
        bool there[2];  // (behind the last page id is -1)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            slot[j] = (p0 + 4 * (i + j)) * 16;
            there[j] = held(id[j]);
        }
        if constexpr (!WHOLE && NEW) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (fresh && there[j] && slot[j] + 16 > u.ctx) take_new_tokens<H>(u, slot[j], lane, sm.stage, k[j], v[j]);
        }
        floatx4 s[2][NT];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int n = 0; n < NT; ++n) s[j][n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < ST; ++st)
#pragma unroll
            for (int w = 0; w < NP; ++w)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int n = 0; n < NT; ++n) s[j][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j][st], qf[n][w][st], s[j][n], 0, 0, 0);
        if (WHOLE || i + 2 < count) refill_k();
        const bool both = there[0] && there[1];
        uint2v p[2][NT][NW];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (!WHOLE || !both) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    bool ok[4];
                    if constexpr (WHOLE) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) ok[e] = there[j];
                    } else {
                        seen_keys(a, c[n].row, base, there[j] ? c[n].limit : -1, slot[j] + kq * 4, ok);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][n][e] = ok[e] ? s[j][n][e] : -INFINITY;
                }
            }
            // The weights are 2^(score - mx) with mx a maximum that is raised only where a score passes it by 2^kSlack: the sums and the
            // output, which a raise multiplies, are then left alone in nearly every round, and no weight exceeds 2^kSlack.
            float pmax = s[0][n][0];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) pmax = fmaxf(pmax, s[j][n][e]);
            if (__ballot(pmax * a.scale > mx[n] + kSlack)) {
                const float mnew = fmaxf(mx[n], max_across_rows(pmax * a.scale));
                const float alpha = __builtin_amdgcn_exp2f(mx[n] - (mnew == -INFINITY ? 0.f : mnew));
                mx[n] = mnew;
                sum[n] *= alpha;
#pragma unroll
                for (int t = 0; t < HT; ++t) o[n][t] *= alpha;
            }
            const float mref = mx[n] == -INFINITY ? 0.f : mx[n];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float x0 = __builtin_amdgcn_exp2f(fmaf(s[j][n][e], a.scale, -mref));
                    const float x1 = __builtin_amdgcn_exp2f(fmaf(s[j][n][e + 1], a.scale, -mref));
                    sum[n] += x0 + x1;  // (of this lane's keys; the four lanes of a column are added up at the end)
                    uint32_t pair[NW];
                    split_pair<NW>(x0, x1, pair);
#pragma unroll
                    for (int q = 0; q < NW; ++q) p[j][n][q][e / 2] = pair[q];
                }
        }
        if (!WHOLE || !both) {  // slots that are not the sequence's may hold anything: not multiplied, not even by zero
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint2v own = first_of_four(there[j] ? u.len - slot[j] - kq * 4 : 0);
#pragma unroll
                for (int t = 0; t < HT; ++t) v[j][t] &= own;
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < NW; ++q)
#pragma unroll
                for (int t = 0; t < HT; ++t)
#pragma unroll
                    for (int n = 0; n < NT; ++n) o[n][t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(short4v, v[j][t]), __builtin_bit_cast(short4v, p[j][n][q]), o[n][t], 0, 0, 0);
        if (WHOLE || i + 2 < count) refill_v(i + 2);
    };
    // (loads return in order: the queries, needed in every round, before the first pages)
    __builtin_amdgcn_sched_barrier(0);
    if (count > 0) {
        next_id[0] = page_id(0);
        next_id[1] = page_id(1);
        refill_k();
        refill_v(0);
    }
    if constexpr (NEW) {
        if (fresh)
            each_new_token<H, T>(a, u, kvh, u.ctx, u.len, [&](int slot, int c, bf16x8 wk, bf16x8 wv) {
                const int t = slot - u.ctx;
                *reinterpret_cast<bf16x8*>(&sm.stage.k[t][c * 8]) = wk;
#pragma unroll
                for (int i = 0; i < 8; ++i) sm.stage.v[c * 8 + i][(u.ctx & 3) + t] = wv[i];
                if (slot >= own0 && slot < own1) store_token<H>(a, u, kvh, slot, c, wk, wv);
            });
    }
    int i = 0;
    if (count > 0)
        for (; i < plain; i += 2) round(i, std::true_type{});
    if (NEW && fresh) __syncthreads();
    if (count > 0)
        for (; i < count; i += 2) round(i, std::false_type{});
    if (NEW && fresh) __syncthreads();  // (the results meet where the new tokens were)
    // tile by tile: the wavefronts' results, then those of the cuts.  A thread has CH elements of a column.
    const int rc = tid >> 4, ch = (tid & 15) * CH;
    constexpr int PART = kPartFloats<H>;
    float* part = a.part + (size_t(blockIdx.x) * a.cuts + cut) * (PART * NT);
    float acc[NT][CH], acc_m[NT], acc_l[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (n > 0) __syncthreads();
        const float l = sum_across_rows(sum[n]);
        if (kq == 0) {
            red_m[wave][col] = mx[n];
            red_l[wave][col] = l;
        }
#pragma unroll
        for (int t = 0; t < HT; ++t) *reinterpret_cast<floatx4*>(&red[wave][col][t * 16 + kq * 4]) = o[n][t];
        __syncthreads();
        const float mg = fmaxf(fmaxf(red_m[0][rc], red_m[1][rc]), fmaxf(red_m[2][rc], red_m[3][rc])), mref = mg == -INFINITY ? 0.f : mg;
        acc_m[n] = mg;
        acc_l[n] = 0.f;
#pragma unroll
        for (int e = 0; e < CH; ++e) acc[n][e] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(red_m[w][rc] - mref);
            acc_l[n] += f * red_l[w][rc];
#pragma unroll
            for (int e = 0; e < CH; ++e) acc[n][e] += f * red[w][rc][ch + e];
        }
    }
    if (uc.n > 1) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (rho0 + n * 16 + rc >= R) continue;
#pragma unroll
            for (int e = 0; e < CH; e += 4)
                *reinterpret_cast<floatx4*>(part + n * PART + rc * H + ch + e) = floatx4{acc[n][e], acc[n][e + 1], acc[n][e + 2], acc[n][e + 3]};
            if (ch == 0) {
                part[n * PART + 16 * H + rc] = acc_m[n];
                part[n * PART + 16 * H + 16 + rc] = acc_l[n];
            }
        }
        return;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const Column rcol = column_of(a, u, kvh, rho0 + n * 16 + rc);
        if (!rcol.ok) continue;
        const float inv = acc_l[n] == 0.f ? 0.f : 1.0f / acc_l[n];
        T* to = static_cast<T*>(a.out) + int64_t(rcol.row) * a.o_row + int64_t(rcol.head) * a.o_head + ch;
#pragma unroll
        for (int e = 0; e < CH; ++e) to[e] = static_cast<T>(acc[n][e] * inv);
    }
}

// For many rows: 128 rows x heads of a KV head at a time, 32 per wavefront, two pages per round.  Every page is fetched once per workgroup and goes
// through LDS: K as it lies, V with the two pages side by side, so that 16 bytes of a lane are its operand of a matrix instruction over 32
// tokens.  A round's phases depend on each other, and a compute unit holds two workgroups, so the rounds overlap: while the
// weights of round i are taken (vector units), the matrix units make the scores of round i + 1; the pages of round i + 2 go to LDS, those of
// i + 3 are on their way to registers.  Three buffers, one barrier per round.  Per round a wavefront issues 52 matrix instructions, 832 clocks, and 138
// vector instructions, 16 of them exponentials, and LDS is busy for 640 clocks of a workgroup; two rounds take 2750.  2000 rows x 4 behind 14000
// tokens, 8 KV heads of 128: 492 GFLOP in 655 us, 0.75 PFLOP/s, with the second part of the weights 738 GFLOP of products, 1.13, where a large bf16
// product reaches 1.25 here; the matrix units are busy 52 % of the time at 2.1 GHz.  64 rows per wavefront, which would halve the LDS reads,
// leave a compute unit one workgroup and nothing to overlap with (with weights in one part 507 -> 995).
constexpr int kManyWaves = 4, kManyTiles = 2 * kManyWaves;  // tiles of 16 rows x heads of a workgroup
template <int H>
__global__ __launch_bounds__(256, 2) void k_attend_many(AttendArgs a) {
    using T = __bf16;
    constexpr int NW = kWeightParts<T>;
    constexpr int ST = H / 32, HT = H / 16, UNITS = ST * 64;  // UNITS: 16 bytes each of a page of one head
    constexpr int PER = UNITS * 2 / 256;                      // of K, and of V, of a thread per round
    __shared__ uint4v sk[3][2][UNITS], sv[3][HT * 64];
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, kq = lane >> 4, cut = blockIdx.y;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kvh = blockIdx.x % uint32_t(a.Hkv);
    const int at_unit = (gridDim.x - 1 - blockIdx.x) / uint32_t(a.Hkv);  // the last rows, which see most, first
    const SeqUnit u = find_unit(a, at_unit, a.G, 16 * kManyTiles, 1);
    const int R = u.n_new * a.G, rho0 = u.index * 16 * kManyTiles;
    if (u.index < 0 || rho0 >= R) return;
    const UnitCuts uc = cuts_of(a, u, (min(rho0 + 16 * kManyTiles, R) - 1) / a.G);
    if (cut >= uc.n) return;
    const int p0 = __builtin_amdgcn_readfirstlane(cut * uc.pages);
    const int p1 = __builtin_amdgcn_readfirstlane(min(uc.all_pages, (cut + 1) * uc.pages));
    const int base = a.mask ? max(a.mask_base[u.seq], 0) : 0;
    // the wavefront's rows: slots below all_see are seen by each of them
    const int rw = rho0 + wave * 32;
    const int all_see = __builtin_amdgcn_readfirstlane(a.mask ? min(base, u.len) : min(u.ctx + min(rw, R - 1) / a.G + 1, u.len));
    Column c[2];
    bf16x8 qf[2][1][ST];
    floatx4 o[2][HT];
    floatx4 sum[2];  // of the weights: a product with ones
    float mx[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        c[n] = column_of(a, u, kvh, rw + n * 16 + col);
        load_query<H, T, 1>(a, c[n], kq, qf[n]);
#pragma unroll
        for (int t = 0; t < HT; ++t) o[n][t] = floatx4{0.f, 0.f, 0.f, 0.f};
        mx[n] = -INFINITY;
        sum[n] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const int32_t* table = a.tables + int64_t(u.seq) * a.table_pages;
    // page ids, a lane each: 64 in use, the next 64 under way
    int ids = p0 + lane < p1 ? table[p0 + lane] : -1, ids_next = p0 + 64 + lane < p1 ? table[p0 + 64 + lane] : -1;
    const int rounds = (p1 - p0 + 1) >> 1;
    const auto held_bit = [&](int id) { return id >= 0 && id < a.n_pages ? 1 : 0; };
    // a thread's share of a round's pages: the same units of both, or (half as many units) one of either
    uint4v rk[PER], rv[PER];
    int got = 0;  // which of the fetched pages are there, a bit each
    const auto fetch = [&](int i) {
        if (i > 0 && (i & 31) == 0) {
            ids = ids_next;
            ids_next = p0 + 2 * i + 64 + lane < p1 ? table[p0 + 2 * i + 64 + lane] : -1;
        }
        const int id0 = __builtin_amdgcn_readlane(ids, 2 * i & 63), id1 = __builtin_amdgcn_readlane(ids, (2 * i + 1) & 63);
        got = held_bit(id0) | held_bit(id1) << 1;
        const size_t at0 = (size_t(got & 1 ? id0 : 0) * a.Hkv + kvh) * (16 * H), at1 = (size_t(got & 2 ? id1 : 0) * a.Hkv + kvh) * (16 * H);
        if constexpr (PER == 2) {
            rk[0] = reinterpret_cast<const uint4v*>(a.kpool + at0)[tid];
            rk[1] = reinterpret_cast<const uint4v*>(a.kpool + at1)[tid];
            rv[0] = reinterpret_cast<const uint4v*>(a.vpool + at0)[tid];
            rv[1] = reinterpret_cast<const uint4v*>(a.vpool + at1)[tid];
        } else {
            const size_t at = wave >= 2 ? at1 : at0;
            rk[0] = reinterpret_cast<const uint4v*>(a.kpool + at)[tid & 127];
            rv[0] = reinterpret_cast<const uint4v*>(a.vpool + at)[tid & 127];
        }
    };
    // What was fetched for round i goes to buffer b.  Slots that are not the sequence's may hold anything: not multiplied, not even by zero.
    const auto put = [&](int i, int b) {
        const int slot0 = (p0 + 2 * i) * 16;
        const bool ragged = got != 3 || slot0 + 32 > u.len;
        if constexpr (PER == 2) {
            sk[b][0][tid] = rk[0];
            sk[b][1][tid] = rk[1];
            uint4v w0 = rv[0], w1 = rv[1];
            if (ragged) {
                const int slot = slot0 + ((tid & 63) >> 4) * 4;
                const uint2v m0 = first_of_four(got & 1 ? u.len - slot : 0), m1 = first_of_four(got & 2 ? u.len - slot - 16 : 0);
                w0 &= uint4v{m0[0], m0[1], m0[0], m0[1]};
                w1 &= uint4v{m1[0], m1[1], m1[0], m1[1]};
            }
            const int at = (tid >> 6) * 128 + (tid & 63);
            sv[b][at] = uint4v{w0[0], w0[1], w1[0], w1[1]};
            sv[b][at + 64] = uint4v{w0[2], w0[3], w1[2], w1[3]};
        } else {
            const int page = wave >> 1, unit = tid & 127;
            sk[b][page][unit] = rk[0];
            uint4v w = rv[0];
            if (ragged) {
                const uint2v m = first_of_four(got & (1 << page) ? u.len - slot0 - page * 16 - ((unit & 63) >> 4) * 4 : 0);
                w &= uint4v{m[0], m[1], m[0], m[1]};
            }
            uint2v* to = reinterpret_cast<uint2v*>(&sv[b][(unit >> 6) * 128 + (unit & 63)]) + page;
            to[0] = uint2v{w[0], w[1]};
            to[128] = uint2v{w[2], w[3]};
        }
    };
    const bf16x8 ones = __builtin_bit_cast(bf16x8, uint4v{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
    bf16x8 k[2][ST];
    const auto take_k = [&](int b) {
#pragma unroll
        for (int st = 0; st < ST; ++st) {
            k[0][st] = __builtin_bit_cast(bf16x8, sk[b][0][st * 64 + lane]);
            k[1][st] = __builtin_bit_cast(bf16x8, sk[b][1][st * 64 + lane]);
        }
    };
    const auto make_scores = [&](floatx4 (&s)[2][2]) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int n = 0; n < 2; ++n) s[j][n] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < ST; ++st)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int n = 0; n < 2; ++n) s[j][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j][st], qf[n][0][st], s[j][n], 0, 0, 0);
    };
    int held, held_next;  // of the pages of this round, of the next one
    floatx4 s[2][2];
    fetch(0);
    held = got;
    put(0, 0);
    fetch(1);  // (pages behind the last one: not there)
    held_next = got;
    put(1, 1);
    fetch(2);
    __syncthreads();
    take_k(0);
    make_scores(s);
    take_k(1);
    int b = 0;
    for (int i = 0; i < rounds; ++i) {
        const int slot0 = (p0 + 2 * i) * 16, b1 = b == 2 ? 0 : b + 1, b2 = b1 == 2 ? 0 : b1 + 1;
        put(i + 2, b2);  // (read last before the barrier of the round before)
        const int held_2 = got;
        fetch(i + 3);
        if (held != 3 || slot0 + 32 > all_see) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    bool ok[4];
                    seen_keys(a, c[n].row, base, held & (1 << j) ? c[n].limit : -1, slot0 + j * 16 + kq * 4, ok);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][n][e] = ok[e] ? s[j][n][e] : -INFINITY;
                }
        }
        float pmax[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            pmax[n] = s[0][n][0];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) pmax[n] = fmaxf(pmax[n], s[j][n][e]);
            pmax[n] *= a.scale;
        }
        if (__ballot(pmax[0] > mx[0] + kSlack || pmax[1] > mx[1] + kSlack)) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float mnew = fmaxf(mx[n], max_across_rows(pmax[n]));
                const float alpha = __builtin_amdgcn_exp2f(mx[n] - (mnew == -INFINITY ? 0.f : mnew));
                mx[n] = mnew;
                sum[n] *= alpha;
#pragma unroll
                for (int t = 0; t < HT; ++t) o[n][t] *= alpha;
            }
        }
        bf16x8 v[HT];
#pragma unroll
        for (int t = 0; t < HT; ++t) v[t] = __builtin_bit_cast(bf16x8, sv[b][t * 64 + lane]);
        floatx4 s1[2][2];
        make_scores(s1);  // of the next round (behind the last one: of nothing, and not used)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const float mref = mx[n] == -INFINITY ? 0.f : mx[n];
            uint4v w[NW];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    uint32_t pair[NW];
                    const float x0 = __builtin_amdgcn_exp2f(fmaf(s[j][n][e], a.scale, -mref));
                    const float x1 = __builtin_amdgcn_exp2f(fmaf(s[j][n][e + 1], a.scale, -mref));
                    split_pair<NW>(x0, x1, pair);
#pragma unroll
                    for (int q = 0; q < NW; ++q) w[q][j * 2 + e / 2] = pair[q];
                }
            // The products of a tile stay together, in front of the other workgroup's instructions: 2000 rows x 4 behind 14000 tokens 649 us,
            // without the priority 704, left to the compiler's order 690.
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int q = 0; q < NW; ++q) {
                sum[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, __builtin_bit_cast(bf16x8, w[q]), sum[n], 0, 0, 0);
#pragma unroll
                for (int t = 0; t < HT; ++t)
                    o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[t], __builtin_bit_cast(bf16x8, w[q]), o[n][t], 0, 0, 0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int n = 0; n < 2; ++n) s[j][n] = s1[j][n];
        held = held_next;
        held_next = held_2;
        __syncthreads();
        b = b1;
        take_k(b2);
    }
    float* part = a.part + ((size_t(at_unit) * a.Hkv + kvh) * a.cuts + cut) * (kPartFloats<H> * kManyTiles) + wave * 2 * kPartFloats<H>;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        if (!c[n].ok) continue;
        const float l = sum[n][0];
        if (uc.n > 1) {
            float* to = part + n * kPartFloats<H>;
#pragma unroll
            for (int t = 0; t < HT; ++t) *reinterpret_cast<floatx4*>(to + col * H + t * 16 + kq * 4) = o[n][t];
            if (kq == 0) {
                to[16 * H + col] = mx[n];
                to[16 * H + 16 + col] = l;
            }
            continue;
        }
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        T* to = static_cast<T*>(a.out) + int64_t(c[n].row) * a.o_row + int64_t(c[n].head) * a.o_head + kq * 4;
#pragma unroll
        for (int t = 0; t < HT; ++t) {
            const floatx4 x = o[n][t] * inv;
            *reinterpret_cast<uint2v*>(to + t * 16) = uint2v{pack_pair(x[0], x[1]), pack_pair(x[2], x[3])};
        }
    }
}

// Adds up what the cuts of a unit left.  One workgroup: four columns of a tile, sixteen threads each, four times over: every fourth cut, of which the
// results of four are under way together.  The sums are taken in an order that the number of cuts fixes.
template <int H, typename T, int NT>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a) {
    constexpr int CH = H / 16, PART = kPartFloats<H>, GROUP = 4;
    __shared__ float red[4][4][16][CH + 2];
    const SeqUnit u = find_unit(a, blockIdx.x / uint32_t(a.Hkv), a.G, 16 * NT, 1);
    const int R = u.n_new * a.G, rho0 = u.index * 16 * NT, n = blockIdx.y >> 2;
    if (u.index < 0 || rho0 + n * 16 + (blockIdx.y & 3) * 4 >= R) return;
    const UnitCuts uc = cuts_of(a, u, (min(rho0 + 16 * NT, R) - 1) / a.G);
    if (uc.n == 1) return;
    const int tid = threadIdx.x, quarter = tid >> 6, at = tid & 15, cl = tid >> 4 & 3, rc = (blockIdx.y & 3) * 4 + cl, ch = at * CH;
    const int rho = rho0 + n * 16 + rc;
    const float* first = a.part + size_t(blockIdx.x) * a.cuts * (PART * NT) + n * PART;
    float mg = -INFINITY, lg = 0.f, acc[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) acc[e] = 0.f;
    if (rho < R)
        for (int s0 = quarter; s0 < uc.n; s0 += 4 * GROUP) {
            float m[GROUP], l[GROUP];
            floatx4 w[GROUP][CH / 4];
#pragma unroll
            for (int g = 0; g < GROUP; ++g) {
                const float* from = first + size_t(min(s0 + 4 * g, uc.n - 1)) * (PART * NT);
                m[g] = s0 + 4 * g < uc.n ? from[16 * H + rc] : -INFINITY;
                l[g] = from[16 * H + 16 + rc];
#pragma unroll
                for (int e = 0; e < CH / 4; ++e) w[g][e] = *reinterpret_cast<const floatx4*>(from + rc * H + ch + e * 4);
            }
            float mnew = mg;
#pragma unroll
            for (int g = 0; g < GROUP; ++g) mnew = fmaxf(mnew, m[g]);
            const float mref = mnew == -INFINITY ? 0.f : mnew, old = __builtin_amdgcn_exp2f(mg - mref);
            lg *= old;
#pragma unroll
            for (int e = 0; e < CH; ++e) acc[e] *= old;
#pragma unroll
            for (int g = 0; g < GROUP; ++g) {
                const float f = __builtin_amdgcn_exp2f(m[g] - mref);
                lg += f * l[g];
#pragma unroll
                for (int e = 0; e < CH; ++e) acc[e] += f * w[g][e / 4][e % 4];
            }
            mg = mnew;
        }
#pragma unroll
    for (int e = 0; e < CH; ++e) red[quarter][cl][at][e] = acc[e];
    red[quarter][cl][at][CH] = mg;
    red[quarter][cl][at][CH + 1] = lg;
    __syncthreads();
    const Column c = column_of(a, u, blockIdx.x % uint32_t(a.Hkv), rho);
    if (quarter != 0 || !c.ok) return;
#pragma unroll
    for (int q = 1; q < 4; ++q) mg = fmaxf(mg, red[q][cl][at][CH]);
    const float mref = mg == -INFINITY ? 0.f : mg;
    lg = 0.f;
#pragma unroll
    for (int e = 0; e < CH; ++e) acc[e] = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float f = __builtin_amdgcn_exp2f(red[q][cl][at][CH] - mref);
        lg += f * red[q][cl][at][CH + 1];
#pragma unroll
        for (int e = 0; e < CH; ++e) acc[e] += f * red[q][cl][at][e];
    }
    const float inv = lg == 0.f ? 0.f : 1.0f / lg;
    T* to = static_cast<T*>(a.out) + int64_t(c.row) * a.o_row + int64_t(c.head) * a.o_head + ch;
#pragma unroll
    for (int e = 0; e < CH; ++e) to[e] = static_cast<T>(acc[e] * inv);
}

}  // namespace card
