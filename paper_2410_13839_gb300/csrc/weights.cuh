// weights.cuh -- the work of a key weights call, for both of its kernels (key_weights.cu,
// key_weights_tc.cu).
//
// The query heads that share a key head are rows of one product: row p of a slot and key
// head is token p / G, query head h G + p % G (G = heads per key head).  The product is made
// with the keys as its rows, S^T = K Q^T, so that a key's weight, the sum over the rows that see
// it, adds up in one thread (or four lanes).  Every key of a slot and key head belongs to one CTA;
// nothing is shared but the rows of long chunks, whose segments' sums a second kernel adds in order.
#pragma once
#include "serving.cuh"

namespace mtp {

constexpr int KW_MAX_SLOTS = 4096;
constexpr float LOG2E = 1.4426950408889634f;

struct WeightsArgs {
    const uint16_t *q, *pool;
    const int *block_table, *cu_rows, *kv_lens;
    const float* lse;
    float* weights;               // the layer's, slot 0, key head 0
    long long q_stride, w_slot;   // elements between rows, between slots' weights
    int slots, rows, kv_heads, group, dim, page_shift, bt_stride, n_pages, width;
    int page_blocks, layer_block;  // (layer, K | V, head) blocks of a page; the layer's first
    int window, max_new, keys;     // keys: of a slot at most
    int tiles;                     // of 128 keys that a CTA of the tensor-core kernel has: 1 or 4
    int segments;                  // row segments of the tensor-core kernel; > 1: sums into `part`
    float* part;                   // [segments][slots][kv_heads][width]
    bool q_vec;                    // rows 16-byte aligned
    float scale_log2;              // scale * log2 e
    int* err;
};

// A slot: its first row, new tokens (as far as they lie in the row buffers), the position of the first of them, its length.
struct WeightsSlot {
    int row0, n, base, len;
};
// `cut` is set where rows that cu_rows gives the slot do not lie in the buffers, where they are more than max_new, where a slot with new tokens
// has more keys than max_keys, and where its length has no place in the table: such a slot has no key.
__device__ __forceinline__ WeightsSlot weights_slot(const WeightsArgs& a, int s, bool& cut) {
    WeightsSlot x;
    x.row0 = a.cu_rows[s];
    const int end = a.cu_rows[s + 1], given = a.kv_lens[s];
    const bool placed = x.row0 >= 0 && end >= x.row0, held = given >= 0 && given <= a.width;
    x.len = held ? given : 0;
    x.n = placed ? max(0, min(end, a.rows) - x.row0) : 0;
    x.base = placed ? max(x.len - (end - x.row0), -(1 << 22)) : 0;  // (rows of positions below 0 see no key)
    cut = !placed || end > a.rows || (x.n > 0 && (!held || x.len > a.keys)) || x.n > a.max_new;
    x.n = min(x.n, a.max_new);
    return x;
}

// Tokens [x, y) of a slot that see a key of [key0, key1).
__device__ __forceinline__ int2 seeing(const WeightsArgs& a, const WeightsSlot& s, int key0, int key1) {
    const int from = max(0, key0 - s.base), last = s.base + s.n - 1;
    int to = s.n;
    if (a.window > 0 && last >= key1 - 1 + a.window) to = key1 - 1 + a.window - s.base;  // positions below key1 - 1 + window
    return make_int2(from, max(from, to));
}

cudaError_t launch_weights_tc(const WeightsArgs& a, const CUtensorMap& map, const CUtensorMap& q_map, bool q_tma, int dtype,
                              int key_tiles, cudaStream_t s);

}  // namespace mtp
