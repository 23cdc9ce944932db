// Page copies and slot moves inside the page pools.
#pragma once
#include "card_common.hip"

namespace card {

// The lists travel by value: a captured graph keeps them, and no upload stands in front of the kernel.
constexpr int kCopyPairs = 224, kMoveSlots = 480;

struct CopyArgs {
    uint4v* pool[2];
    size_t layer16;   // 16-byte units of a layer of a pool
    int32_t page16;   // of a page
    int32_t src[kCopyPairs], dst[kCopyPairs];
};

// One workgroup: one page of one layer of one pool.  Bound by memory: 157 pages of 32 layers x 8 heads x 128, 659 MB, in 126 us, 5.2 TB/s.
__global__ __launch_bounds__(256) void k_kv_copy_pages(CopyArgs a) {
    uint4v* base = a.pool[blockIdx.z] + blockIdx.y * a.layer16;
    const uint4v* from = base + size_t(a.src[blockIdx.x]) * a.page16;
    uint4v* to = base + size_t(a.dst[blockIdx.x]) * a.page16;
    for (int i = threadIdx.x; i < a.page16; i += 256) to[i] = from[i];
}

struct MoveArgs {
    __bf16* kpool;
    __bf16* vpool;
    size_t layer_elems;
    int32_t n, part, n_kv_heads;  // part: moves of a workgroup (of all that may touch each other's slots there is one)
    int32_t src[kMoveSlots], dst[kMoveSlots];  // (dst -1: not a move, see below)
};

// Tokens between slots.  Bound by memory: a token is 2 h bytes of K in pieces of 16 and 2 h of V in pieces of 2, which lie with the same elements of
// its three neighbours.  One workgroup: one head of one layer; a wavefront per 64 elements of K (8 tokens per load) and per 32 elements of V (2
// tokens per load).  A wavefront owns its elements for all moves, and a wavefront's accesses to an address happen in the order of its
// instructions: reading ROUND moves before writing any is the order of the list as long as no move reads what an earlier one
// wrote, and so is reading the next ROUND while these are written.  No barrier, and two rounds under way.  The host puts gaps into the list so that
// slots that go to four neighbours in a row begin at a multiple of four.
// 1500 tokens of 32 layers x 8 heads x 128, closing gaps of 600 between them, us: a move at a time, a thread per element, 720; rounds of 96
// moves 125 in the kernels (471 MB with the gaps' share of the lines: 3.8 TB/s), 138 a call of four launches.
// Rounds of 32 for short lists, which are a matter of latency: 128 moves in rounds of 32 and of 96 12.6 and 14.6, 192 17.7 and 20.7, 256 21.8 and
// 20.8, 1500 136 and 124 (of 64, 128 moves: 1500 128, 129; 128 14.8, 18.8); 16 layers, 192 12.4 and 14.6, 256 15.6 and 14.1, 1500 91 and 74.
constexpr int kMoveRound = 96, kMoveShort = 32;
constexpr int kMoveApart = kMoveShort;  // moves of a workgroup of a list that needs no order
template <int H, int ROUND>
__global__ __launch_bounds__(H / 64 * 192) void k_kv_move_slots(MoveArgs a) {
    typedef __attribute__((ext_vector_type(2))) unsigned int uint2v;
    constexpr int LISTS = (ROUND + 63) / 64;  // registers of a lane that hold a round's slots
    const int head = blockIdx.x, lane = threadIdx.x & 63, first = blockIdx.z * a.part, end = min(a.n, first + a.part);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const auto page_at = [&](int slot) { return (size_t(slot >> 4) * a.n_kv_heads + head) * (16 * H); };
    // the slots of the round from move i on, a lane each; behind the end the last one once more, which is not written
    const auto fetch = [&](const int32_t* list, int i, int (&v)[LISTS]) {
#pragma unroll
        for (int l = 0; l < LISTS; ++l) v[l] = list[min(i + l * 64 + lane, end - 1)];
    };
    // rounds in turn: the next one is read before this one is written
    const auto all = [&](auto& v, auto&& read, auto&& write) {
        int to[2][LISTS];
        read(first, v[0], to[0]);
        for (int i = first; i < end; i += 2 * ROUND) {
            if (i + ROUND < end) read(i + ROUND, v[1], to[1]);
            write(i, v[0], to[0]);
            if (i + ROUND >= end) break;
            if (i + 2 * ROUND < end) read(i + 2 * ROUND, v[0], to[0]);
            write(i + ROUND, v[1], to[1]);
        }
    };
    if (wave < H / 64) {  // K: 8 elements of 8 tokens
        constexpr int N = ROUND / 8;
        __bf16* pool = a.kpool + blockIdx.y * a.layer_elems;
        const int group = wave * 8 + (lane & 7), tok = lane >> 3;
        const auto place = [&](int slot) { return reinterpret_cast<uint4v*>(pool + page_at(slot) + (group * 16 + (slot & 15)) * 8); };
        uint4v v[2][N];
        all(v,
            [&](int i, uint4v (&w)[N], int (&d)[LISTS]) {
                int s[LISTS];
                fetch(a.src, i, s);
                fetch(a.dst, i, d);
#pragma unroll
                for (int r = 0; r < N; ++r) w[r] = *place(__shfl(s[r / 8], r % 8 * 8 + tok));
            },
            [&](int i, const uint4v (&w)[N], const int (&d)[LISTS]) {
#pragma unroll
                for (int r = 0; r < N; ++r) {
                    const int slot = __shfl(d[r / 8], r % 8 * 8 + tok);
                    if (i + r * 8 + tok < end && slot >= 0) *place(slot) = w[r];
                }
            });
        return;
    }
    // V: an element of 2 tokens, of the tokens that lie together as far as they go to four such places
    constexpr int N = ROUND / 2;
    unsigned short* pool = reinterpret_cast<unsigned short*>(a.vpool + blockIdx.y * a.layer_elems);
    const int half = lane >> 5, elem = v_page_index((wave - H / 64) * 32 + (lane & 31), 0);
    const auto place = [&](int slot) { return pool + page_at(slot) + (slot & 15) / 4 * 128 + (slot & 3) + elem; };
    unsigned short v[2][N];
    all(v,
        [&](int i, unsigned short (&w)[N], int (&d)[LISTS]) {
            int s[LISTS];
            fetch(a.src, i, s);
            fetch(a.dst, i, d);
            // (a lane's tokens: four in a row, then the other half's four)
#pragma unroll
            for (int r = 0; r < N; ++r) {
                const int at = r / 4 * 8 + r % 4, x = __builtin_amdgcn_readlane(s[at / 64], at % 64), y = __builtin_amdgcn_readlane(s[at / 64], at % 64 + 4);
                w[r] = *place(half ? y : x);
            }
        },
        [&](int i, const unsigned short (&w)[N], const int (&d)[LISTS]) {
#pragma unroll
            for (int r = 0; r < N; r += 4) {
                const int at = r * 2 + half * 4;
                int to[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int x = __builtin_amdgcn_readlane(d[r * 2 / 64], r * 2 % 64 + e), y = __builtin_amdgcn_readlane(d[r * 2 / 64], r * 2 % 64 + 4 + e);
                    to[e] = half ? y : x;
                }
                // (a list that ends inside the four repeats its last slot: not in a row)
                if (to[0] % 4 == 0 && to[1] == to[0] + 1 && to[2] == to[0] + 2 && to[3] == to[0] + 3) {
                    *reinterpret_cast<uint2v*>(place(to[0])) = uint2v{w[r] | uint32_t(w[r + 1]) << 16, w[r + 2] | uint32_t(w[r + 3]) << 16};
                    continue;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + at + e < end && to[e] >= 0) *place(to[e]) = w[r + e];
            }
        });
}

}  // namespace card
