// Attention of the new tokens of a ragged batch over one paged cache of 4 bits a value (Page4).
//
// With a token's scale s and offset b of each 64 channels g, and its codes c: k q = sum_g s_g (sum (16 + c) q) + b_g (sum q), and sum p v = sum (p s_g)(16 + c) + sum p b_g.
// So the matrix instructions take 16 + c, exact in bf16, for keys and values; scores are put together from a sum per group, weights enter the product with values once per
// group, multiplied by its scales, and the offsets' part is one number a row and group.
#pragma once
#include "card_append.hip"

namespace card {

// Numbers that are kept from the compiler: it would write the first two into two instructions where registers make one, and the third as a constant that the product takes
// for another one.
struct InRegisters {
    uint32_t mask = 0x00780078u, sixteen = 0x41804180u, minus_first = 0x0000bf80u, minus_second = 0xbf800000u;
    __device__ __forceinline__ InRegisters() { asm("" : "+s"(mask), "+v"(sixteen), "+s"(minus_first), "+s"(minus_second)); }
    // 16 + c of the codes in bits 4 R .. + 3 of either half of a word, as bf16.
    template <int R>
    __device__ __forceinline__ uint32_t pair(uint32_t w) const {
        return ((R == 0 ? w << 3 : w >> (4 * R - 3)) & mask) | sixteen;
    }
    __device__ __forceinline__ uint4v pairs(uint32_t w) const { return uint4v{pair<0>(w), pair<1>(w), pair<2>(w), pair<3>(w)}; }
    // Two floats as sums of N bf16, as split_pair gives them: what the first part leaves comes out of a product with it, (-1, 0) and (0, -1), exact and an instruction each.
    template <int N>
    __device__ __forceinline__ void split(float x0, float x1, uint32_t (&p)[N]) const {
        typedef __attribute__((ext_vector_type(2))) float float2v;
        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bf16x2 part = __builtin_convertvector((float2v{x0, x1}), bf16x2);
            p[i] = __builtin_bit_cast(uint32_t, part);
            if (i + 1 < N) {
                x0 = __builtin_amdgcn_fdot2_f32_bf16(part, __builtin_bit_cast(bf16x2, minus_first), x0, false);
                x1 = __builtin_amdgcn_fdot2_f32_bf16(part, __builtin_bit_cast(bf16x2, minus_second), x1, false);
            }
        }
    }
};
__device__ __forceinline__ uint32_t centred(uint32_t pair) {  // less 24: c - 8
    const float x = __uint_as_float(pair << 16) - 24.f, y = __uint_as_float(pair & 0xffff0000u) - 24.f;
    return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
}

// A lane's share of a page: of K the codes of token col, channels 32 st + 8 kq .. + 7 in word st; of V those of tokens 4 kq .. + 3, channels 64 g + col + 16 r, in words
// [token / 2][g]; and of the words one, from which the sixteen lanes of a row have what belongs to their four tokens: lane 8 kind + 4 g + e the word of
// token 4 kq + e and group g of K (0) or V (1).  (H = 64: 4 kind + e.)  The lanes that need it take it as an operand that is broadcast inside the row.
template <int H>
struct Codes4 {
    static constexpr int N = H / 32, G = H / 64;
    uint32_t k[N], v[N];
};
template <int H>
constexpr __host__ __device__ int word_lane(int kind, int g, int e) { return kind * (H / 16) + g * 4 + e; }
template <int I>
__device__ __forceinline__ float row_lane(uint32_t v) {
    return __uint_as_float(uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x150 | I, 0xf, 0xf, true)));
}
template <int N>
__device__ __forceinline__ void load_words(const char* p, uint32_t (&w)[N]) {
    if constexpr (N == 4) {
        const uint4v x = *reinterpret_cast<const uint4v*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = x[i];
    } else {
        const uint2v x = *reinterpret_cast<const uint2v*>(p);
        w[0] = x[0];
        w[1] = x[1];
    }
}
// f(std::integral_constant) for 0 .. N - 1.
template <int N, typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) { each_of<N>(f, std::make_integer_sequence<int, N>{}); }

// With fp32 rows sums keep to small numbers: codes enter as c - 8, with the offset of code 8 in place of b, and each round's products with values are added up on their
// own.  (Otherwise a sum of products and its offsets are some 24 scales each, and nearly cancel.)
constexpr float kMiddle = 24.f;

// Sums of a row's query over the channels of each group, of the parts that the products take.
template <int H, int NP>
__device__ __forceinline__ void query_sums(const bf16x8 (&qf)[NP][H / 32], float (&qs)[H / 64]) {
#pragma unroll
    for (int g = 0; g < H / 64; ++g) {
        float s = 0.f;
#pragma unroll
        for (int st = 2 * g; st < 2 * g + 2; ++st)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float x = static_cast<float>(qf[NP - 1][st][e]);
#pragma unroll
                for (int w = NP - 2; w >= 0; --w) x += static_cast<float>(qf[w][st][e]);
                s += x;
            }
        qs[g] = sum_across_rows(s);
    }
}
// The scores of tokens 4 kq .. + 3 from the products of their groups; and weights times scales, and times offsets, of tokens 4 kq .. + 3 and one group.  Broadcasts are operands
// of the instructions, which the compiler makes moves of: 16 instructions instead of 32 a page.  (The compiler does not count for them: what is broadcast must be two
// instructions old, a matrix instruction of four passes has its result after 8 and has read its registers after 3.)
template <int H>
__device__ __forceinline__ void scores_of(const floatx4 (&acc)[H / 64], const float (&qs)[H / 64], uint32_t scales, uint32_t offsets, float (&s)[4]) {
    if constexpr (H == 128) {
        asm("s_nop 7\n"  //
            "v_mul_f32_dpp %0, %4, %6 row_newbcast:0 row_mask:0xf bank_mask:0xf\n"
            "v_mul_f32_dpp %1, %4, %7 row_newbcast:1 row_mask:0xf bank_mask:0xf\n"
            "v_mul_f32_dpp %2, %4, %8 row_newbcast:2 row_mask:0xf bank_mask:0xf\n"
            "v_mul_f32_dpp %3, %4, %9 row_newbcast:3 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %0, %4, %10 row_newbcast:4 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %1, %4, %11 row_newbcast:5 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %2, %4, %12 row_newbcast:6 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %3, %4, %13 row_newbcast:7 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %0, %5, %14 row_newbcast:0 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %1, %5, %14 row_newbcast:1 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %2, %5, %14 row_newbcast:2 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %3, %5, %14 row_newbcast:3 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %0, %5, %15 row_newbcast:4 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %1, %5, %15 row_newbcast:5 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %2, %5, %15 row_newbcast:6 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %3, %5, %15 row_newbcast:7 row_mask:0xf bank_mask:0xf"
            : "=&v"(s[0]), "=&v"(s[1]), "=&v"(s[2]), "=&v"(s[3])
            : "v"(scales), "v"(offsets), "v"(acc[0][0]), "v"(acc[0][1]), "v"(acc[0][2]), "v"(acc[0][3]), "v"(acc[1][0]), "v"(acc[1][1]), "v"(acc[1][2]),
              "v"(acc[1][3]), "v"(qs[0]), "v"(qs[1]));
    } else {
        asm("s_nop 7\n"
            "v_mul_f32_dpp %0, %4, %6 row_newbcast:0 row_mask:0xf bank_mask:0xf\n"
            "v_mul_f32_dpp %1, %4, %7 row_newbcast:1 row_mask:0xf bank_mask:0xf\n"
            "v_mul_f32_dpp %2, %4, %8 row_newbcast:2 row_mask:0xf bank_mask:0xf\n"
            "v_mul_f32_dpp %3, %4, %9 row_newbcast:3 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %0, %5, %10 row_newbcast:0 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %1, %5, %10 row_newbcast:1 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %2, %5, %10 row_newbcast:2 row_mask:0xf bank_mask:0xf\n"
            "v_fmac_f32_dpp %3, %5, %10 row_newbcast:3 row_mask:0xf bank_mask:0xf"
            : "=&v"(s[0]), "=&v"(s[1]), "=&v"(s[2]), "=&v"(s[3])
            : "v"(scales), "v"(offsets), "v"(acc[0][0]), "v"(acc[0][1]), "v"(acc[0][2]), "v"(acc[0][3]), "v"(qs[0]));
    }
}
template <int AT>  // (the lane of token 4 kq's word)
__device__ __forceinline__ void scaled_weights(const float (&p)[4], uint32_t scales, uint32_t offsets, float (&w)[4], float& sum) {
    asm("s_nop 3\n"
        "v_mul_f32_dpp %0, %5, %7 row_newbcast:%c11 row_mask:0xf bank_mask:0xf\n"
        "v_mul_f32_dpp %1, %5, %8 row_newbcast:%c12 row_mask:0xf bank_mask:0xf\n"
        "v_mul_f32_dpp %2, %5, %9 row_newbcast:%c13 row_mask:0xf bank_mask:0xf\n"
        "v_mul_f32_dpp %3, %5, %10 row_newbcast:%c14 row_mask:0xf bank_mask:0xf\n"
        "v_fmac_f32_dpp %4, %6, %7 row_newbcast:%c11 row_mask:0xf bank_mask:0xf\n"
        "v_fmac_f32_dpp %4, %6, %8 row_newbcast:%c12 row_mask:0xf bank_mask:0xf\n"
        "v_fmac_f32_dpp %4, %6, %9 row_newbcast:%c13 row_mask:0xf bank_mask:0xf\n"
        "v_fmac_f32_dpp %4, %6, %10 row_newbcast:%c14 row_mask:0xf bank_mask:0xf"
        : "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]), "+v"(sum)
        : "v"(scales), "v"(offsets), "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "n"(AT), "n"(AT + 1), "n"(AT + 2), "n"(AT + 3));
}

// 16 NT rows x heads of a KV head at a time.  One workgroup: one cut of the pages of a sequence, for one KV head; its four wavefronts take every fourth page each, two per
// round, and refill K as soon as the scores are done, V behind P V.  Bound by vector instructions: a round of two pages is 278 of them (558 as the compiler makes them
// of the same formulas, see InRegisters and scores_of), 128 to make operands of codes, which two tiles share, and some 150 a tile; and 24 matrix instructions a tile.  64 texts of 800-8000
// tokens, a row of 4 heads each, 334 MB, in 84 us (4.0 TB/s; vector units busy 56 % of the time, matrix units 14; loads alone 70); 5 rows x 8 behind 120000 tokens 69;
// 2000 rows x 4 behind 14000 1000, 0.49 PFLOP/s, with the second part of the weights 0.74.  Four pages per round with two wavefronts per SIMD 105 for the 64 texts,
// with three, spilling, 148.  A kernel for many rows whose wavefronts share pages made operands in LDS (two tiles a wavefront, four wavefronts) took 950 for the
// 2000 rows, but 44 for 500 rows behind 300 tokens against 22 and 257 for three texts of up to 1000 rows x 7 against 229.
template <int H, typename T, int NT>
__global__ __launch_bounds__(256, NT * sizeof(T) == 2 ? 3 : 2) void k_attend4(AttendArgs a) {
    constexpr int ST = H / 32, HT = H / 16, NP = sizeof(T) == 4 ? 3 : 1, NW = kWeightParts<T>, LD = H + 4, CH = H / 16, G = H / 64, ROUND = 2;
    constexpr bool FINE = sizeof(T) == 4;
    using P4 = Page4<H>;
    __shared__ __align__(16) float red[4][16][LD];  // (written as floatx4)
    __shared__ float red_m[4][16], red_l[4][16];
    static_assert(__alignof__(red) % 16 == 0 && LD % 4 == 0, "");
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, kq = lane >> 4, cut = blockIdx.y;
    const int kvh = blockIdx.x % uint32_t(a.Hkv), at_unit = blockIdx.x / uint32_t(a.Hkv);
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const SeqUnit u = find_unit(a, at_unit, a.G, 16 * NT, 1);
    const int R = u.n_new * a.G, rho0 = u.index * 16 * NT;
    if (u.index < 0 || rho0 >= R) return;
    const int m_first = rho0 / a.G, m_last = (min(rho0 + 16 * NT, R) - 1) / a.G;
    const UnitCuts uc = cuts_of(a, u, m_last);
    if (cut >= uc.n) return;
    const int p0 = __builtin_amdgcn_readfirstlane(cut * uc.pages + wave), p1 = __builtin_amdgcn_readfirstlane(min(uc.all_pages, (cut + 1) * uc.pages));
    const int base = a.mask ? max(a.mask_base[u.seq], 0) : 0;
    const int all_see = __builtin_amdgcn_readfirstlane(a.mask ? min(base, u.len) : min(u.ctx + m_first + 1, u.len));  // slots below are seen by every row
    Column c[NT];
    bf16x8 qf[NT][NP][ST];
    floatx4 o[NT][HT];
    float mx[NT], sum[NT], qs[NT][G], bs[NT][G];  // bs: of the weights times offsets
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        c[n] = column_of(a, u, kvh, rho0 + n * 16 + col);
        load_query<H, T, NP>(a, c[n], kq, qf[n]);
        query_sums<H, NP>(qf[n], qs[n]);
#pragma unroll
        for (int i = 0; i < HT; ++i) o[n][i] = floatx4{0.f, 0.f, 0.f, 0.f};
        mx[n] = -INFINITY;
        sum[n] = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) bs[n][g] = 0.f;
    }
    const const_i32* ids = reinterpret_cast<const const_i32*>(reinterpret_cast<uintptr_t>(a.tables + int64_t(u.seq) * a.table_pages));
    const int count = p0 < p1 ? (p1 - p0 + 3) >> 2 : 0;
    const auto page_id = [&](int i) { return i < count ? ids[p0 + 4 * i] : -1; };
    const auto held = [&](int id) { return id >= 0 && id < a.n_pages; };
    const int plain_end = min(p1, min(all_see, u.len) >> 4);  // pages below are seen whole by every row
    const int plain = min(p0 < plain_end ? (plain_end - p0 + 3) >> 2 : 0, count - ROUND) / ROUND * ROUND;
    const int place = col & 3;  // the lane's word: of which of the row's tokens, and where
    const int kind = col / (H / 16) & 1;
    const char* word_pool = reinterpret_cast<const char*>(kind ? a.vpool : a.kpool) + P4::kCodes + ((col >> 2 & (G - 1)) * 16 + kq * 4 + place) * 4;
    const char* k_pool = reinterpret_cast<const char*>(a.kpool) + lane * (ST * 4);
    const char* v_pool = reinterpret_cast<const char*>(a.vpool) + lane * (ST * 4);
    const InRegisters bits;
    Codes4<H> x[ROUND];
    uint32_t next_word[ROUND];
    int id[ROUND], next_id[ROUND];
    const auto refill_k = [&]() {
#pragma unroll
        for (int j = 0; j < ROUND; ++j) {
            id[j] = next_id[j];
            const size_t at = P4::at(held(id[j]) ? id[j] : 0, a.Hkv, kvh);
            load_words(k_pool + at, x[j].k);
            next_word[j] = *reinterpret_cast<const uint32_t*>(word_pool + at);
        }
    };
    const auto refill_v = [&](int i) {
#pragma unroll
        for (int j = 0; j < ROUND; ++j) load_words(v_pool + P4::at(held(id[j]) ? id[j] : 0, a.Hkv, kvh), x[j].v);
#pragma unroll
        for (int j = 0; j < ROUND; ++j) next_id[j] = page_id(i + ROUND + j);
    };
    const auto round = [&](int i, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        int slot[ROUND];
        bool there[ROUND], all = true;
        uint32_t word[ROUND], scale[ROUND], offset[ROUND];
#pragma unroll
        for (int j = 0; j < ROUND; ++j) {
            slot[j] = (p0 + 4 * (i + j)) * 16;
            there[j] = held(id[j]);
            all = all && there[j];
            word[j] = next_word[j];
        }
        if (!WHOLE || !all) {  // places that are not the sequence's may hold anything: zero
#pragma unroll
            for (int j = 0; j < ROUND; ++j) word[j] = there[j] && slot[j] + kq * 4 + place < u.len ? word[j] : 0u;
        }
#pragma unroll
        for (int j = 0; j < ROUND; ++j) {
            scale[j] = word[j] << 16;
            offset[j] = FINE ? __float_as_uint(fmaf(__uint_as_float(scale[j]), kMiddle, __uint_as_float(word[j]))) : word[j];
        }
        float s[ROUND][NT][4];
        uint32_t ok = 0xffffffffu;  // of the lane's keys, a bit each: [NT][ROUND][4]
#pragma unroll
        for (int j = 0; j < ROUND; ++j) {
            floatx4 acc[NT][G];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int g = 0; g < G; ++g) acc[n][g] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < ST; ++y) {  // (the groups in turn: products of one wait for each other)
                const int st = y % G * 2 + y / G;
                uint4v codes = bits.pairs(x[j].k[st]);
                if constexpr (FINE) codes = uint4v{centred(codes[0]), centred(codes[1]), centred(codes[2]), centred(codes[3])};
                const bf16x8 k = __builtin_bit_cast(bf16x8, codes);
#pragma unroll
                for (int w = 0; w < NP; ++w)
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[n][st / 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[n][w][st], acc[n][st / 2], 0, 0, 0);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) scores_of<H>(acc[n], qs[n], scale[j], offset[j], s[j][n]);
            __builtin_amdgcn_sched_barrier(0);  // (pages one after the other: together they do not fit the registers)
        }
        if (WHOLE || i + ROUND < count) refill_k();
        if (!WHOLE || !all) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < ROUND; ++j) {
                    bool on[4];
                    if constexpr (WHOLE) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) on[e] = there[j];
                    } else {
                        seen_keys(a, c[n].row, base, there[j] ? c[n].limit : -1, slot[j] + kq * 4, on);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[j][n][e] = on[e] ? s[j][n][e] : -INFINITY;
                        if (!on[e]) ok &= ~(1u << ((n * ROUND + j) * 4 + e));
                    }
                }
        }
        // (weights are taken as in k_attend_few, with their slack)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float pmax = s[0][n][0];
#pragma unroll
            for (int j = 0; j < ROUND; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) pmax = fmaxf(pmax, s[j][n][e]);
            if (__ballot(pmax * a.scale > mx[n] + kSlack)) {
                const float mnew = fmaxf(mx[n], max_across_rows(pmax * a.scale));
                const float alpha = __builtin_amdgcn_exp2f(mx[n] - (mnew == -INFINITY ? 0.f : mnew));
                mx[n] = mnew;
                sum[n] *= alpha;
#pragma unroll
                for (int g = 0; g < G; ++g) bs[n][g] *= alpha;
#pragma unroll
                for (int t = 0; t < HT; ++t) o[n][t] *= alpha;
            }
            const float mref = mx[n] == -INFINITY ? 0.f : mx[n];
#pragma unroll
            for (int j = 0; j < ROUND; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[j][n][e] = __builtin_amdgcn_exp2f(fmaf(s[j][n][e], a.scale, -mref));
                    sum[n] += s[j][n][e];
                }
        }
        floatx4 turn[FINE ? NT : 1][FINE ? HT : 1];
        if constexpr (FINE) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < HT; ++t) turn[n][t] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
        auto& to = [&]() -> auto& { if constexpr (FINE) return turn; else return o; }();
#pragma unroll
        for (int j = 0; j < ROUND; j += 2)
            each<G>([&](auto g) {
                uint4v p[NT][NW];
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    each<2>([&](auto b) {
                        constexpr int B = decltype(b)::value, AT = word_lane<H>(1, decltype(g)::value, 0);
                        float w[4];
                        if constexpr (WHOLE) {
                            scaled_weights<AT>(s[j + B][n], scale[j + B], offset[j + B], w, bs[n][g]);
                        } else {  // (a hidden token's scale may be NaN: it is not multiplied, not even by zero)
                            each<4>([&](auto e) {
                                constexpr int E = decltype(e)::value;
                                const bool on = ok >> ((n * ROUND + j + B) * 4 + E) & 1u;
                                const float p = s[j + B][n][E], ws = p * row_lane<AT + E>(scale[j + B]), wb = p * row_lane<AT + E>(offset[j + B]);
                                w[E] = on ? ws : 0.f;
                                bs[n][g] += on ? wb : 0.f;
                            });
                        }
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            uint32_t pair[NW];
                            bits.split(w[e], w[e + 1], pair);
#pragma unroll
                            for (int q = 0; q < NW; ++q) p[n][q][B * 2 + e / 2] = pair[q];
                        }
                    });
                bf16x8 v[4];
                each<4>([&](auto r) {
                    constexpr int RR = decltype(r)::value;
                    uint4v codes = {bits.template pair<RR>(x[j].v[g]), bits.template pair<RR>(x[j].v[G + g]), bits.template pair<RR>(x[j + 1].v[g]), bits.template pair<RR>(x[j + 1].v[G + g])};
                    if constexpr (FINE) codes = uint4v{centred(codes[0]), centred(codes[1]), centred(codes[2]), centred(codes[3])};
                    v[RR] = __builtin_bit_cast(bf16x8, codes);
                });
#pragma unroll
                for (int q = 0; q < NW; ++q)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            to[n][g * 4 + r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[r], __builtin_bit_cast(bf16x8, p[n][q]), to[n][g * 4 + r], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            });
        if constexpr (FINE) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int t = 0; t < HT; ++t) o[n][t] += turn[n][t];
        }
        if (WHOLE || i + ROUND < count) refill_v(i + ROUND);
    };
    __builtin_amdgcn_sched_barrier(0);  // (the queries, needed in every round, before the first pages)
    if (count > 0) {
#pragma unroll
        for (int j = 0; j < ROUND; ++j) next_id[j] = page_id(j);
        refill_k();
        refill_v(0);
        int i = 0;
        for (; i < plain; i += ROUND) round(i, std::true_type{});
        for (; i < count; i += ROUND) round(i, std::false_type{});
    }
    // tile by tile: the wavefronts' results, then those of the cuts.  A thread has CH elements of a column.
    const int rc = tid >> 4, ch = (tid & 15) * CH;
    constexpr int PART = kPartFloats<H>;
    float* part = a.part + (size_t(blockIdx.x) * a.cuts + cut) * (PART * NT);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (n > 0) __syncthreads();
        const float l = sum_across_rows(sum[n]);
        if (kq == 0) {
            red_m[wave][col] = mx[n];
            red_l[wave][col] = l;
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float b = sum_across_rows(bs[n][g]);
#pragma unroll
            for (int t = g * 4; t < g * 4 + 4; ++t) *reinterpret_cast<floatx4*>(&red[wave][col][t * 16 + kq * 4]) = o[n][t] + b;
        }
        __syncthreads();
        const float mg = fmaxf(fmaxf(red_m[0][rc], red_m[1][rc]), fmaxf(red_m[2][rc], red_m[3][rc])), mref = mg == -INFINITY ? 0.f : mg;
        float acc[CH], total = 0.f;
#pragma unroll
        for (int e = 0; e < CH; ++e) acc[e] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(red_m[w][rc] - mref);
            total += f * red_l[w][rc];
#pragma unroll
            for (int e = 0; e < CH; ++e) acc[e] += f * red[w][rc][ch + e];
        }
        const Column rcol = column_of(a, u, kvh, rho0 + n * 16 + rc);
        if (!rcol.ok) continue;
        if (uc.n > 1) {
#pragma unroll
            for (int e = 0; e < CH; e += 4) *reinterpret_cast<floatx4*>(part + n * PART + rc * H + ch + e) = floatx4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
            if (ch == 0) {
                part[n * PART + 16 * H + rc] = mg;
                part[n * PART + 16 * H + 16 + rc] = total;
            }
            continue;
        }
        const float inv = total == 0.f ? 0.f : 1.0f / total;
        T* to = static_cast<T*>(a.out) + int64_t(rcol.row) * a.o_row + int64_t(rcol.head) * a.o_head + ch;
#pragma unroll
        for (int e = 0; e < CH; ++e) to[e] = static_cast<T>(acc[e] * inv);
    }
}

}  // namespace card
