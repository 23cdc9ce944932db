// Page copies and slot moves inside the page pools.
#pragma once
#include "card_common.hip"

namespace card {

// The lists travel by value: a captured graph keeps them, and no upload stands in front of the kernel.
constexpr int kCopyPairs = 224, kMoveSlots = 448;

struct CopyArgs {
    uint4v* pool[2];
    size_t layer16;   // 16-byte units of a layer of a pool
    int32_t page16;   // of a page
    int32_t src[kCopyPairs], dst[kCopyPairs];
};

// One workgroup: one page of one layer of one pool.
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
    int32_t n, n_kv_heads, head_dim;
    int32_t src[kMoveSlots], dst[kMoveSlots];
};

// One workgroup: one head of one layer, a thread per head element, the moves in order.
__global__ __launch_bounds__(128) void k_kv_move_slots(MoveArgs a) {
    const int head = blockIdx.x, j = threadIdx.x, h = a.head_dim;
    if (j >= h) return;
    __bf16* k = a.kpool + blockIdx.y * a.layer_elems;
    __bf16* v = a.vpool + blockIdx.y * a.layer_elems;
    for (int i = 0; i < a.n; ++i) {
        const int s = a.src[i], d = a.dst[i];
        const size_t from = (size_t(s >> 4) * a.n_kv_heads + head) * (16 * h), to = (size_t(d >> 4) * a.n_kv_heads + head) * (16 * h);
        k[to + ((j >> 3) * 16 + (d & 15)) * 8 + (j & 7)] = k[from + ((j >> 3) * 16 + (s & 15)) * 8 + (j & 7)];
        v[to + v_page_index(j, d & 15)] = v[from + v_page_index(j, s & 15)];
    }
}

}  // namespace card
