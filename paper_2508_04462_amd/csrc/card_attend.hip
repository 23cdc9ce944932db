// Attention of the new tokens of a ragged batch over one paged cache.
#pragma once
#include "card_common.hip"

namespace card {

typedef __attribute__((ext_vector_type(2))) unsigned int uint2v;

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
    // the pages of a sequence in up to `cuts` cuts of cut_pages or more; where there are several: their partial results and how many have
    // arrived, per unit and KV head (counters; cleared by the kernel that stores the keys)
    int32_t cuts, cut_pages, counters;
    float* part;
    uint32_t* arrived;
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

// Clears the arrival counters; keys and values of the new tokens go to their pages.  One workgroup: one page of one KV head.  A thread writes the 8 elements of a token
// that lie together in K, or the 4 tokens of an element that lie together in V.
constexpr int kStoreUnits = 2;  // pages per sequence beyond its new tokens / 16
template <typename T>
__global__ __launch_bounds__(256) void k_attend_store(AttendArgs a, int h) {
    for (int i = (blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x; i < a.counters; i += gridDim.x * gridDim.y * 256) a.arrived[i] = 0u;
    if (!a.k) return;
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
    for (int st = 0; st < H / 32; ++st)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            __bf16 w[NP];
            split_parts<NP>(static_cast<float>(p[st * 32 + e]), w);
#pragma unroll
            for (int i = 0; i < NP; ++i) qf[i][st][e] = w[i];
        }
}
template <int H>
__device__ __forceinline__ void load_k_page(const AttendArgs& a, int id, int kvh, int lane, bf16x8 (&k)[H / 32]) {
    const bf16x8* p = reinterpret_cast<const bf16x8*>(a.kpool + (size_t(id) * a.Hkv + kvh) * (16 * H)) + lane;
#pragma unroll
    for (int st = 0; st < H / 32; ++st) k[st] = p[st * 64];
}
template <int H>
__device__ __forceinline__ void load_v_page(const AttendArgs& a, int id, int kvh, int lane, short4v (&v)[H / 16]) {
    const uint4v* p = reinterpret_cast<const uint4v*>(a.vpool + (size_t(id) * a.Hkv + kvh) * (16 * H)) + lane;
#pragma unroll
    for (int i = 0; i < H / 32; ++i) {
        const uint4v w = p[i * 64];
        v[2 * i] = __builtin_bit_cast(short4v, uint2v{w[0], w[1]});
        v[2 * i + 1] = __builtin_bit_cast(short4v, uint2v{w[2], w[3]});
    }
}

constexpr int kAuxDev = 16;  // device scope
__device__ __forceinline__ __amdgpu_buffer_rsrc_t dev_rsrc(const void* base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, 0xffffffffu, 0x00020000);
}

// For few rows per sequence (16 NT rows x heads of a KV head at a time): bound by reading the cache, so every page is read once, straight into
// the registers that the matrix instructions take it from.  One workgroup: one cut of the pages of a sequence, for one KV head; its four
// wavefronts take every fourth page each, two per round, and refill K as soon as the scores are done, V behind P V.  The wavefronts' results
// meet in LDS, the cuts' in memory: the last one to arrive adds them up, in their order.
template <int H, typename T, int NT>
__global__ __launch_bounds__(256, NT * sizeof(T) == 2 ? 3 : (NT * sizeof(T) == 4 ? 2 : 1)) void k_attend_few(AttendArgs a) {
    constexpr int ST = H / 32, HT = H / 16, NP = sizeof(T) == 4 ? 3 : 1, LD = H + 4, CH = H / 16;
    __shared__ __align__(16) float red[4][16][LD];
    __shared__ float red_m[4][16], red_l[4][16];
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, kq = lane >> 4, kvh = blockIdx.y, cut = blockIdx.z;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const SeqUnit u = find_unit(a, blockIdx.x, a.G, 16 * NT, 1);
    const int R = u.n_new * a.G, rho0 = u.index * 16 * NT;
    if (u.index < 0 || rho0 >= R) return;
    // the pages that the last of the rows sees, and this cut's part of them
    const int m_first = rho0 / a.G, m_last = (min(rho0 + 16 * NT, R) - 1) / a.G;
    const int n_keys = a.mask ? u.len : min(u.ctx + m_last + 1, u.len);
    const int n_pages = (n_keys + 15) >> 4;
    const int per_cut = max(a.cut_pages, (n_pages + a.cuts - 1) / a.cuts), n_cuts = (n_pages + per_cut - 1) / per_cut;
    if (cut >= n_cuts) return;
    const int p0 = cut * per_cut + wave, p1 = min(n_pages, cut * per_cut + per_cut);
    const int base = a.mask ? max(a.mask_base[u.seq], 0) : 0;
    const int all_see = a.mask ? min(base, u.len) : min(u.ctx + m_first + 1, u.len);  // slots below are seen by every row
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
    const int32_t* table = a.tables + int64_t(u.seq) * a.table_pages;
    int ids = 0;  // of this wavefront's pages, 64 at a time, a lane each
    const auto page_id = [&](int i) { return __builtin_amdgcn_readlane(ids, i & 63); };
    const int count = p0 < p1 ? (p1 - p0 + 3) >> 2 : 0;
    const auto fetch_ids = [&](int i) { ids = i + lane < count ? table[p0 + 4 * (i + lane)] : -1; };
    const auto held = [&](int id) { return id >= 0 && id < a.n_pages; };
    bf16x8 k[2][ST];
    short4v v[2][HT];
    int id[2];
    if (count > 0) {
        fetch_ids(0);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            id[j] = page_id(j);
            load_k_page<H>(a, held(id[j]) ? id[j] : 0, kvh, lane, k[j]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) load_v_page<H>(a, held(id[j]) ? id[j] : 0, kvh, lane, v[j]);
    }
    for (int i = 0; i < count; i += 2) {
        int slot[2];
        bool there[2], full = true;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            slot[j] = (p0 + 4 * (i + j)) * 16;
            there[j] = held(id[j]);  // (behind the last page id is -1)
            full = full && there[j] && slot[j] + 16 <= all_see;
        }
        short4v p[2][NT][NP];
        float alpha[NT];
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
        if (i + 2 < count) {
            if (((i + 2) & 63) == 0) fetch_ids(i + 2);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                id[j] = page_id(i + 2 + j);
                load_k_page<H>(a, held(id[j]) ? id[j] : 0, kvh, lane, k[j]);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (!full) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    bool ok[4];
                    seen_keys(a, c[n].row, base, there[j] ? c[n].limit : -1, slot[j] + kq * 4, ok);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][n][e] = ok[e] ? s[j][n][e] : -INFINITY;
                }
            }
            float pmax = -INFINITY;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[j][n][e] *= a.scale;
                    pmax = fmaxf(pmax, s[j][n][e]);
                }
            const float mnew = fmaxf(mx[n], max_across_rows(pmax)), mref = mnew == -INFINITY ? 0.f : mnew;
            alpha[n] = __builtin_amdgcn_exp2f(mx[n] - mref);
            mx[n] = mnew;
            float psum = 0.f;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = __builtin_amdgcn_exp2f(s[j][n][e] - mref);
                    psum += x;
                    __bf16 w[NP];
                    split_parts<NP>(x, w);
#pragma unroll
                    for (int q = 0; q < NP; ++q) p[j][n][q][e] = __builtin_bit_cast(short, w[q]);
                }
            sum[n] = sum[n] * alpha[n] + psum;  // (of this lane's keys; the four lanes of a column are added up at the end)
        }
        if (!full) {  // slots that are not the sequence's may hold anything: not multiplied, not even by zero
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int own = there[j] ? u.len - slot[j] - kq * 4 : 0;
#pragma unroll
                for (int t = 0; t < HT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[j][t][e] = e < own ? v[j][t][e] : short(0);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int t = 0; t < HT; ++t) o[n][t] *= alpha[n];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < NP; ++q)
#pragma unroll
                for (int t = 0; t < HT; ++t)
#pragma unroll
                    for (int n = 0; n < NT; ++n) o[n][t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v[j][t], p[j][n][q], o[n][t], 0, 0, 0);
        if (i + 2 < count) {
#pragma unroll
            for (int j = 0; j < 2; ++j) load_v_page<H>(a, held(id[j]) ? id[j] : 0, kvh, lane, v[j]);
        }
    }
    // tile by tile: the wavefronts' results, then those of the cuts.  A thread has CH elements of a column.
    const int rc = tid >> 4, ch = (tid & 15) * CH;
    const size_t unit = size_t(blockIdx.x) * a.Hkv + kvh;
    constexpr int PART = 16 * (H + 2);  // floats that a cut leaves per tile: [16][H], [16] maxima, [16] sums
    float* part = a.part + (unit * a.cuts + cut) * (PART * NT);
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
    if (n_cuts > 1) {
        const __amdgpu_buffer_rsrc_t rs = dev_rsrc(part);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (rho0 + n * 16 + rc < R) {
#pragma unroll
                for (int e = 0; e < CH; e += 4) {
                    const floatx4 w = {acc[n][e], acc[n][e + 1], acc[n][e + 2], acc[n][e + 3]};
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4v, w), rs, (n * PART + rc * H + ch + e) * 4, 0, kAuxDev);
                }
                if (ch == 0) {
                    st_agent(part + n * PART + 16 * H + rc, acc_m[n]);
                    st_agent(part + n * PART + 16 * H + 16 + rc, acc_l[n]);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (tid == 0) last = __hip_atomic_fetch_add(&a.arrived[unit], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == uint32_t(n_cuts) - 1;
        __syncthreads();
        if (!last) return;
        const float* first = a.part + unit * a.cuts * (PART * NT);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (rho0 + n * 16 + rc >= R) continue;
            float mg = -INFINITY, lg = 0.f;
#pragma unroll
            for (int e = 0; e < CH; ++e) acc[n][e] = 0.f;
            constexpr int GROUP = 8;  // cuts whose results are under way together
            for (int s0 = 0; s0 < n_cuts; s0 += GROUP) {
                float m[GROUP], l[GROUP];
                uint4v w[GROUP][CH / 4];
#pragma unroll
                for (int g = 0; g < GROUP; ++g) {
                    const float* from = first + size_t(min(s0 + g, n_cuts - 1)) * (PART * NT) + n * PART;
                    m[g] = ld_agent(from + 16 * H + rc);
                    l[g] = ld_agent(from + 16 * H + 16 + rc);
                    const __amdgpu_buffer_rsrc_t rf = dev_rsrc(from);
#pragma unroll
                    for (int e = 0; e < CH / 4; ++e) w[g][e] = __builtin_amdgcn_raw_buffer_load_b128(rf, (rc * H + ch + e * 4) * 4, 0, kAuxDev);
                }
                float mnew = mg;
#pragma unroll
                for (int g = 0; g < GROUP; ++g) mnew = fmaxf(mnew, m[g]);
                const float mref = mnew == -INFINITY ? 0.f : mnew, old = __builtin_amdgcn_exp2f(mg - mref);
                lg *= old;
#pragma unroll
                for (int e = 0; e < CH; ++e) acc[n][e] *= old;
#pragma unroll
                for (int g = 0; g < GROUP; ++g) {
                    const float f = s0 + g < n_cuts ? __builtin_amdgcn_exp2f(m[g] - mref) : 0.f;
                    lg += f * l[g];
#pragma unroll
                    for (int e = 0; e < CH; ++e) acc[n][e] += f * __uint_as_float(w[g][e / 4][e % 4]);
                }
                mg = mnew;
            }
            acc_l[n] = lg;
        }
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

}  // namespace card
