// Rotation of the queries and keys of a ragged batch, and the storing of keys and values to pages of 16 or of 4 bits a value; what a
// cache of 4 bits holds, read back.
#pragma once
#include "card_attend.hip"

namespace card {

// ---- the cache in 4 bits -------------------------------------------------------------------------------
// A page of one KV head: 8 H bytes of codes, then a word for each 64 channels of a token, [H / 64][16 tokens].  The lower half of a word is a
// scale in bf16, the whole word in fp32 an offset, and code c stands for scale * (16 + c) + offset: 4.5 bits a value.  16 + c is a bf16 with the
// code in bits 3-6, which a shift and one more instruction make of two codes, so the matrix instructions take codes, and scales and offsets come to
// their sums.  Codes lie as the instructions take them, from the lowest bits on: K [4][16 tokens][H / 32][2][4], which are channel / 8 % 4, token,
// channel / 32, channel % 2, channel % 8 / 2; V [4][16][2][H / 64][2][4], which are token / 4, channel % 16, token / 2 % 2, channel / 64, token % 2,
// channel / 16 % 4: a lane's share of a page is 16 bytes of either (H = 128), a pair of neighbours of an operand lies 16 bits apart.
template <int H>
struct Page4 {
    static constexpr int kCodes = 8 * H, kBytes = 9 * H;
    static __device__ __forceinline__ size_t at(int page, int heads, int head) { return (size_t(page) * heads + head) * kBytes; }
    static __device__ __forceinline__ int k_word(int chunk, int t) { return ((chunk & 3) * 16 + t) * (H / 32) + (chunk >> 2); }  // of channels 8 chunk .. + 7
    static __device__ __forceinline__ int v_half(int col, int group, int t) {  // of channels 64 group + col, + 16, + 32, + 48
        return ((((t >> 2) * 16 + col) * 2 + (t >> 1 & 1)) * (H / 64) + group) * 2 + (t & 1);
    }
    static __device__ __forceinline__ int word(int group, int t) { return kCodes / 4 + group * 16 + t; }
};
__device__ __forceinline__ float scale_of(uint32_t word) { return __uint_as_float(word << 16); }
__device__ __forceinline__ float offset_of(uint32_t word) { return __uint_as_float(word); }

// The word for values from low to high.  The 16 levels reach from below low to above high by what rounding the offset may cost, and the scale is no less
// than 2^-10 of the largest value, so that a group of equal values finds its level, too: a code is off by half a scale at most.
// Every operation is rounded on its own, whatever the compiler could make of two: the same values give the same word anywhere.
__device__ __forceinline__ uint32_t word_for(float low, float high, float not_finite) {
#pragma clang fp contract(off)
    const float most = fmaxf(-low, high);
    const float range = (high - low) * (17.f / 256.f), floor = most * (1.f / 1024.f);
    const __bf16 scale = static_cast<__bf16>(range + floor + not_finite);
    const uint32_t bits = bf16_bits(scale);
    const float below = low - most * (1.f / 128.f), sixteen = static_cast<float>(scale) * 16.f;
    return ((__float_as_uint(below - sixteen) - bits + 0x8000u) & 0xffff0000u) | bits;
}
__device__ __forceinline__ uint32_t code_for(float x, uint32_t word, float inverse) {
#pragma clang fp contract(off)
    const float d = x - offset_of(word);
    return uint32_t(fminf(fmaxf(rintf(d * inverse) - 16.f, 0.f), 15.f));
}
__device__ __forceinline__ float inverse_of(uint32_t word) {
    const float s = scale_of(word);
    return s > 0.f ? 1.0f / s : 0.f;
}
__device__ __forceinline__ float value_of(uint32_t code, uint32_t word) { return fmaf(scale_of(word), float(16 + int(code & 15u)), offset_of(word)); }

template <int LANES>  // lowest and highest of LANES neighbouring lanes (4, 8 or 16)
__device__ __forceinline__ void extremes(float& low, float& high) {
    const auto step = [&](auto ctrl) {
        constexpr int C = decltype(ctrl)::value;
        const int l = int(__float_as_uint(low)), h = int(__float_as_uint(high));
        low = fminf(low, __uint_as_float(uint32_t(__builtin_amdgcn_update_dpp(l, l, C, 0xf, 0xf, false))));
        high = fmaxf(high, __uint_as_float(uint32_t(__builtin_amdgcn_update_dpp(h, h, C, 0xf, 0xf, false))));
    };
    step(std::integral_constant<int, 0xB1>{});                             // lane ^ 1
    step(std::integral_constant<int, 0x4E>{});                             // lane ^ 2
    if constexpr (LANES > 4) step(std::integral_constant<int, 0x141>{});   // mirrored in eight
    if constexpr (LANES > 8) step(std::integral_constant<int, 0x140>{});   // mirrored in sixteen
}
// Sum over the lanes of what is zero for finite values and NaN for others.
template <int LANES>
__device__ __forceinline__ float any_not_finite(float v) {
    v = dpp_add<0x4E>(dpp_add<0xB1>(v));
    if constexpr (LANES > 4) v = dpp_add<0x141>(v);
    if constexpr (LANES > 8) v = dpp_add<0x140>(v);
    return v;
}

// ---- rotation and storing --------------------------------------------------------------------------------
struct AppendArgs {
    AttendArgs a;  // (of q and out, the rows to rotate and where they go; nothing of the softmax)
    const int32_t* positions;
    int32_t rotate;
    double turns[64];  // frequencies / 2 pi
};

// cos and sin of x turns, to fp32.  The angle is reduced in 64 bits to an eighth of a turn, for which the Taylor series up to the 15th power leave 3e-15.  Before that it is off by
// 2^-50 of itself at most: the quotient by 2 pi, 2 pi itself and the product with the position are rounded to 2^-53 each, the model's frequencies, of two powers, to some 2^-51.  So cosines are
// the exact ones' roundings to fp32 but for one in 100 000 at positions up to 30 000, in 11 000 from 10^5 on, in 1500 from 10^6 on (h = 128, base 10^4, computed).
__device__ __forceinline__ void cos_sin(double turns, float& c, float& s) {
    turns -= rint(turns);
    const double quarter = rint(turns * 4.0), x = (turns - quarter * 0.25) * 6.283185307179586476925, y = x * x;
    double p = -1.0 / 1307674368000.0, q = 1.0 / 20922789888000.0;
    p = fma(p, y, 1.0 / 6227020800.0);
    q = fma(q, y, -1.0 / 87178291200.0);
    p = fma(p, y, -1.0 / 39916800.0);
    q = fma(q, y, 1.0 / 479001600.0);
    p = fma(p, y, 1.0 / 362880.0);
    q = fma(q, y, -1.0 / 3628800.0);
    p = fma(p, y, -1.0 / 5040.0);
    q = fma(q, y, 1.0 / 40320.0);
    p = fma(p, y, 1.0 / 120.0);
    q = fma(q, y, -1.0 / 720.0);
    p = fma(p, y, -1.0 / 6.0);
    q = fma(q, y, 1.0 / 24.0);
    p = fma(p * y, x, x);
    q = fma(fma(q, y, -0.5), y, 1.0);
    const int at = int(quarter) & 3;
    const float sn = float(at & 1 ? q : p), cs = float(at & 1 ? p : q);
    s = at & 2 ? -sn : sn;
    c = at == 1 || at == 2 ? -cs : cs;
}

// Eight elements of a row of heads.
template <typename T>
struct Eight {
    uint4v w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < int(sizeof(T)) / 2; ++i) w[i] = reinterpret_cast<const uint4v*>(p)[i];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[0][i] << 16);
                x[2 * i + 1] = __uint_as_float(w[0][i] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i / 4][i % 4]);
        }
    }
};
__device__ __forceinline__ uint4v packed8(const float (&x)[8]) {
    return uint4v{pack_pair(x[0], x[1]), pack_pair(x[2], x[3]), pack_pair(x[4], x[5]), pack_pair(x[6], x[7])};
}
__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) { *reinterpret_cast<uint4v*>(p) = packed8(x); }
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) reinterpret_cast<floatx4*>(p)[i] = floatx4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
}

// The rows of one page of a sequence: token t of the page, t0 <= t < t1, is row row0 + t, at position place0 + t.  Those below `stored` have a place in the sequence's table.
// (Places are counted from the table's end for a sequence that is longer than that; positions are not.)
struct PageRows {
    int32_t slot0, t0, t1, stored, page;
    int64_t row0;
    double place0;
    bool some;
};
__device__ __forceinline__ PageRows rows_of_page(const AttendArgs& a, int unit) {
    const SeqUnit u = find_unit(a, unit, 1, 16, kStoreUnits);
    PageRows r;
    const int pg = (u.ctx >> 4) + u.index, end = u.ctx + u.n_new;
    r.slot0 = pg * 16;
    r.some = u.index >= 0 && r.slot0 < end && u.n_new > 0;
    r.t0 = max(u.ctx - r.slot0, 0);
    r.t1 = min(end - r.slot0, 16);
    r.row0 = int64_t(u.row0) + r.slot0 - u.ctx;
    r.place0 = double(u.held) + (r.slot0 - u.ctx);
    r.stored = 0;
    r.page = -1;
    if (r.some && pg < a.table_pages) {
        r.stored = r.t1;
        r.page = a.tables[int64_t(u.seq) * a.table_pages + pg];
        if (r.page < 0 || r.page >= a.n_pages) r.stored = 0;
    }
    return r;
}

// One workgroup: the rows of one page of a sequence, for one KV head and the query heads that share it.  Angles are the same for all heads: each is
// made once, into LDS, while the rows are on their way.  A thread rotates elements 8 c .. + 7 with their partners half a head further on; products are added in 64 bits,
// which makes a rotated value the rounding of these cosines' exact one, the same wherever it is computed, and costs less than reading it.  Bound by memory for prompts (2000
// rows of 64 + 8 heads of 128, 82 MB, in 16.2 us, 5.1 TB/s, on inputs that are not in a cache 18.4; a row of queries at a time 16.7; keys and queries in workgroups of their
// own 18.6), by latency for few rows (5.0 us).  To 4 bits, about 2280 rows of 28 + 4 heads, 13.5 us: some 600 workgroups, two per compute unit, each a chain of K, V, angles and seven heads' queries.
template <int H, typename T, int BITS>
__global__ __launch_bounds__(256) void k_append(AppendArgs g) {
    const AttendArgs& a = g.a;
    constexpr int C = H / 16;  // pairs of 8 elements of a head
    constexpr int U = sizeof(T) == 2 ? 4 : 2;  // of a thread, under way together
    __shared__ float2 table[16][H / 2];
    const PageRows r = rows_of_page(a, blockIdx.x);
    if (!r.some) return;
    const int tid = threadIdx.x, head = blockIdx.y, n = r.t1 - r.t0;
    // keys: a thread's pair; values: BITS = 16 four tokens of an element, 4 the elements of a token that are 16 apart
    const int kt = r.t0 + tid / C, kc = tid % C;
    const bool has_k = tid < n * C;
    const T* kp = static_cast<const T*>(a.k) + (r.row0 + (has_k ? kt : r.t0)) * a.k_row + int64_t(head) * a.k_head + kc * 8;
    Eight<T> kr[2];
    kr[0].load(kp);
    kr[1].load(kp + H / 2);
    const T* vp = static_cast<const T*>(a.v) + int64_t(head) * a.v_head;
    constexpr int VU = BITS == 16 ? 4 * H / 256 : 1, VN = BITS == 16 ? 4 : H / 16;
    float v[VU][VN];
#pragma unroll
    for (int x = 0; x < VU; ++x)
#pragma unroll
        for (int i = 0; i < VN; ++i) {
            const int e = x * 256 + tid;
            const int t = BITS == 16 ? e / H * 4 + i : tid >> 4, j = BITS == 16 ? e % H : i * 16 + (tid & 15);
            v[x][i] = static_cast<float>(vp[(r.row0 + min(max(t, r.t0), r.t1 - 1)) * a.v_row + j]);
        }
    if (g.rotate) {
        for (int e = tid; e < n * (H / 2); e += 256) {
            const int t = r.t0 + e / (H / 2), j = e % (H / 2);
            const double position = g.positions ? double(g.positions[r.row0 + t]) : r.place0 + t;
            float2 cs;
            cos_sin(position * g.turns[j], cs.x, cs.y);
            table[t][j] = cs;
        }
        __syncthreads();
    }
    const auto rotate = [&](int t, int c, float (&x0)[8], float (&x1)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 cs = table[t][c * 8 + i];
            const double z0 = x0[i], z1 = x1[i], co = cs.x, si = cs.y;
            x0[i] = float(z0 * co - z1 * si);  // (the products are exact: rounded once, fused or not)
            x1[i] = float(z1 * co + z0 * si);
        }
    };
    if (g.rotate && a.q) {
        const T* from = static_cast<const T*>(a.q) + int64_t(head) * a.G * a.q_head;
        T* to = static_cast<T*>(a.out) + int64_t(head) * a.G * a.o_head;
        const int units = n * a.G * C;
        for (int e0 = tid; e0 < units; e0 += 256 * U) {
            Eight<T> x0[U], x1[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = min(e0 + u * 256, units - 1), at = e / C;
                const T* p = from + (r.row0 + r.t0 + at / a.G) * a.q_row + at % a.G * a.q_head + e % C * 8;
                x0[u].load(p);
                x1[u].load(p + H / 2);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = e0 + u * 256, at = e / C, t = r.t0 + at / a.G, c = e % C;
                if (e >= units) break;
                float y0[8], y1[8];
                x0[u].get(y0);
                x1[u].get(y1);
                rotate(t, c, y0, y1);
                T* o = to + (r.row0 + t) * a.o_row + at % a.G * a.o_head + c * 8;
                store8(o, y0);
                store8(o + H / 2, y1);
            }
        }
    }
    if (r.stored == 0) return;
    float k0[8], k1[8];
    kr[0].get(k0);
    kr[1].get(k1);
    if (g.rotate && has_k) rotate(kt, kc, k0, k1);
    if constexpr (BITS == 16) {
        const size_t base = (size_t(r.page) * a.Hkv + head) * (16 * H);
        if (has_k) {
            store8(a.kpool + base + (kc * 16 + kt) * 8, k0);
            store8(a.kpool + base + ((kc + C) * 16 + kt) * 8, k1);
        }
#pragma unroll
        for (int x = 0; x < VU; ++x) {
            const int e = x * 256 + tid, j = e % H, t = e / H * 4;
            __bf16* to = a.vpool + base + v_page_index(j, t);
            if (t >= r.t0 && t + 4 <= r.t1) {
                *reinterpret_cast<uint2v*>(to) = uint2v{pack_pair(v[x][0], v[x][1]), pack_pair(v[x][2], v[x][3])};
                continue;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t + i >= r.t0 && t + i < r.t1) to[i] = static_cast<__bf16>(v[x][i]);
        }
    } else {
        using P = Page4<H>;
        uint32_t* kw = reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(a.kpool) + P::at(r.page, a.Hkv, head));
        char* vbytes = reinterpret_cast<char*>(a.vpool) + P::at(r.page, a.Hkv, head);
        // keys: the first halves of a token's pairs are its group 0 and the second ones group 1 (H = 128), or all of them its only one
        float low[2], high[2], odd[2];
        const float* half[2] = {k0, k1};
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            low[b] = high[b] = half[b][0];
            odd[b] = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                low[b] = fminf(low[b], half[b][i]);
                high[b] = fmaxf(high[b], half[b][i]);
                odd[b] += half[b][i] * 0.f;
            }
        }
        if constexpr (H == 64) {
            low[0] = low[1] = fminf(low[0], low[1]);
            high[0] = high[1] = fmaxf(high[0], high[1]);
            odd[0] = odd[1] = odd[0] + odd[1];
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            extremes<C>(low[b], high[b]);
            odd[b] = any_not_finite<C>(odd[b]);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const uint32_t word = word_for(low[b], high[b], odd[b]);
            const float inverse = inverse_of(word);
            uint32_t codes = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) codes |= code_for(half[b][i], word, inverse) << ((i >> 1) * 4 + (i & 1) * 16);
            if (!has_k) continue;
            kw[P::k_word(kc + b * C, kt)] = codes;
            if (kc == 0 && (H == 128 || b == 0)) kw[P::word(b, kt)] = word;
        }
        const int vt = tid >> 4, col = tid & 15;
#pragma unroll
        for (int b = 0; b < H / 64; ++b) {
            float lo = v[0][4 * b], hi = lo, bad = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo = fminf(lo, v[0][4 * b + i]);
                hi = fmaxf(hi, v[0][4 * b + i]);
                bad += v[0][4 * b + i] * 0.f;
            }
            extremes<16>(lo, hi);
            const uint32_t word = word_for(lo, hi, any_not_finite<16>(bad));
            const float inverse = inverse_of(word);
            uint32_t codes = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) codes |= code_for(v[0][4 * b + i], word, inverse) << (4 * i);
            if (vt < r.t0 || vt >= r.t1) continue;
            reinterpret_cast<unsigned short*>(vbytes)[P::v_half(col, b, vt)] = static_cast<unsigned short>(codes);
            if (col == 0) reinterpret_cast<uint32_t*>(vbytes)[P::word(b, vt)] = word;
        }
    }
}

// What a cache of 4 bits holds of the batch's rows.  One workgroup: the rows of one page of a sequence, for one KV head; rows without a place are not touched.
template <int H, typename T>
__global__ __launch_bounds__(256) void k_read4(AttendArgs a) {
    using P = Page4<H>;
    const PageRows r = rows_of_page(a, blockIdx.x);
    if (!r.some || r.stored == 0) return;
    const int tid = threadIdx.x, head = blockIdx.y, n = r.t1 - r.t0;
    const char* kb = reinterpret_cast<const char*>(a.kpool) + P::at(r.page, a.Hkv, head);
    const char* vb = reinterpret_cast<const char*>(a.vpool) + P::at(r.page, a.Hkv, head);
    const uint32_t *kw = reinterpret_cast<const uint32_t*>(kb), *vw = reinterpret_cast<const uint32_t*>(vb);
    T* ko = static_cast<T*>(const_cast<void*>(a.k)) + int64_t(head) * a.k_head;
    T* vo = static_cast<T*>(const_cast<void*>(a.v)) + int64_t(head) * a.v_head;
    if (tid < n * (H / 8)) {
        const int t = r.t0 + tid / (H / 8), c = tid % (H / 8);
        const uint32_t codes = kw[P::k_word(c, t)], word = kw[P::word(c >> 3, t)];
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = value_of(codes >> ((i >> 1) * 4 + (i & 1) * 16), word);
        store8(ko + (r.row0 + t) * a.k_row + c * 8, x);
    }
    const int t = tid >> 4, col = tid & 15;
    if (t < r.t0 || t >= r.t1) return;
#pragma unroll
    for (int b = 0; b < H / 64; ++b) {
        const uint32_t codes = reinterpret_cast<const unsigned short*>(vb)[P::v_half(col, b, t)], word = vw[P::word(b, t)];
#pragma unroll
        for (int i = 0; i < 4; ++i) vo[(r.row0 + t) * a.v_row + b * 64 + i * 16 + col] = static_cast<T>(value_of(codes >> (4 * i), word));
    }
}

}  // namespace card
