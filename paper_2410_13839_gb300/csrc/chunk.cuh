// chunk.cuh -- the work of a chunk attention call and how it is shared out, for
// both of its kernels (chunk_attention.cu, chunk_attention_tc.cu).
//
// The query heads that share a key head are rows of one product: row p of a slot and
// key head is token p / G, query head h G + p % G (G = heads per key head).  TR
// consecutive rows are a tile; with one key head it is an item.  An item's keys, from the
// first that one of its rows sees to the last, are cut into units of KT keys.  The units
// of all items, item after item, are one stream, of which CTA c of N takes the c-th N-th:
// ragged slots, few long ones or many short ones all give CTAs of equal work, at one
// prologue each.  An item that lies in one CTA's share is written by that CTA.  One that
// several share leaves (maximum, sum, unnormalised output) per row and CTA in the
// workspace, and a merge kernel after this one joins them by their maxima, in the CTAs'
// order: nothing depends on which CTA ends first.
#pragma once
#include "serving.cuh"

namespace mtp {

constexpr int CH_MAX_TILES = 8192, CH_MAX_SLOTS = 4096;

struct ChunkArgs {
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    const int *block_table, *cu_rows, *kv_lens;
    long long q_stride, out_stride;
    int slots, rows, kv_heads, group, page_shift, bt_stride, n_pages;
    uint32_t group_inv;            // ceil(2^32 / group)
    int page_blocks, layer_block;  // (layer, K | V, head) blocks of a page; the layer's first
    int window, max_tiles, min_units;
    int snap;                      // items of at most 1 / snap of a share are not cut (0: all are)
    bool q_vec, out_vec;           // rows 16-byte aligned
    float scale_log2;              // scale * log2 e: scores in log2 units
    float* part;                   // [ctas][2][TR][dim + 2]
    int* desc;                     // [ctas][8]
    int* err;
};

// Token of packed row p: p / group (p < 2^26: the product with the rounded-up inverse has the exact quotient)
__device__ __forceinline__ int chunk_token(const ChunkArgs& a, int p) {
    return a.group == 1 ? p : (int)__umulhi((uint32_t)p, a.group_inv);
}

// Bounded wait for a barrier's phase, as mbar_wait; one short loop, for kernels whose code has to stay
// in the instruction cache.
__device__ __forceinline__ bool chunk_wait(uint64_t* bar, uint32_t parity, int* err) {
#pragma unroll 1
    for (uint32_t i = 0; i < MBAR_MAX_POLLS; ++i)
        if (mbar_try_wait(bar, parity & 1)) return true;
    if (err) atomicOr(err, ERR_WAIT_TIMEOUT);
    return false;
}

struct ChunkTile {
    int slot, row0, n, len;  // the slot, its first row, its new tokens, its length with them
    int p0, rows;            // packed rows [p0, p0 + rows)
    int lo, hi;              // keys [lo, hi) that some row sees (none: hi = lo = 0)
    int key0, units;         // first key of the first unit (a multiple of KT); units, one at least
};

// rows of slot s, as far as they lie in the row buffers
__device__ __forceinline__ void chunk_slot(const ChunkArgs& a, int s, int& row0, int& n) {
    row0 = a.cu_rows[s];
    n = a.cu_rows[s + 1] - row0;
    if (row0 < 0 || row0 > a.rows || n < 0) n = 0;
    n = min(n, a.rows - row0);
}

template <int TR, int KT>
__device__ __forceinline__ ChunkTile chunk_tile(const ChunkArgs& a, int slot, int t) {
    ChunkTile x;
    x.slot = slot;
    chunk_slot(a, slot, x.row0, x.n);
    x.len = max(0, min(a.kv_lens[slot], a.bt_stride << a.page_shift));
    x.p0 = t * TR;
    x.rows = min(x.n * a.group - x.p0, TR);
    const int first = x.len - x.n + chunk_token(a, x.p0), last = x.len - x.n + chunk_token(a, x.p0 + x.rows - 1);  // positions
    x.hi = max(0, last + 1);
    x.lo = a.window > 0 ? min(x.hi, max(0, first - a.window + 1)) : 0;
    x.key0 = x.lo / KT * KT;
    x.units = max(1, (x.hi - x.key0 + KT - 1) / KT);
    return x;
}

struct ChunkMap {
    int* slot_first;       // [slots + 1]: first tile of every slot
    uint32_t* unit_first;  // [tiles + 1]: first unit of every tile, counted for one key head
    int tiles, ctas, snap;
    long long units;       // of all key heads
};
__host__ __device__ inline size_t chunk_map_bytes(int slots, int max_tiles) { return (size_t)(slots + max_tiles + 2) * 4; }

template <class T>
__device__ __forceinline__ int chunk_owner(const T* first, int n, T x) {  // largest i in [0, n) with first[i] <= x
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// The whole block calls it.
template <int WARPS, int TR, int KT>
__device__ __forceinline__ ChunkMap chunk_map(const ChunkArgs& a, void* space, long long (*part)[2]) {
    constexpr int THREADS = WARPS * 32;
    ChunkMap m;
    m.slot_first = static_cast<int*>(space);
    m.unit_first = reinterpret_cast<uint32_t*>(m.slot_first + a.slots + 1);
    long long base = 0, unused = 0, sum, none;
    for (int s0 = 0; s0 < a.slots; s0 += THREADS) {
        const int s = s0 + (int)threadIdx.x;
        long long x = 0;
        if (s < a.slots) {
            int row0, n;
            chunk_slot(a, s, row0, n);
            x = ((long long)n * a.group + TR - 1) / TR;
        }
        block_scan2<WARPS>(x, unused, part, sum, none);
        if (s < a.slots) m.slot_first[s] = (int)min(base + x, (long long)a.max_tiles);
        base += sum;
    }
    m.tiles = (int)min(base, (long long)a.max_tiles);
    if (threadIdx.x == 0) m.slot_first[a.slots] = m.tiles;
    __syncthreads();
    base = 0;
    for (int j0 = 0; j0 < m.tiles; j0 += THREADS) {
        const int j = j0 + (int)threadIdx.x;
        long long x = 0;
        if (j < m.tiles) {
            const int s = chunk_owner(m.slot_first, a.slots, j);
            x = chunk_tile<TR, KT>(a, s, j - m.slot_first[s]).units;
        }
        block_scan2<WARPS>(x, unused, part, sum, none);
        if (j < m.tiles) m.unit_first[j] = (uint32_t)(base + x);
        base += sum;
    }
    if (threadIdx.x == 0) m.unit_first[m.tiles] = (uint32_t)base;
    __syncthreads();
    m.units = base * a.kv_heads;
    m.ctas = (int)min((long long)gridDim.x, max(1ll, (m.units + a.min_units - 1) / a.min_units));
    m.snap = a.snap ? (int)min(m.units / m.ctas / a.snap, 1ll << 30) : 0;
    return m;
}

struct ChunkItem {
    int tile, head;
    long long first;  // its first unit
    int units;
};
static __device__ __noinline__ ChunkItem chunk_item(const ChunkArgs& a, const ChunkMap& m, long long unit) {
    // unit < m.units: unit / kv_heads is a unit of one head
    ChunkItem x;
    x.tile = chunk_owner(m.unit_first, m.tiles, (uint32_t)(unit / a.kv_heads));
    const long long first = (long long)m.unit_first[x.tile] * a.kv_heads;
    x.units = (int)(m.unit_first[x.tile + 1] - m.unit_first[x.tile]);
    x.head = (int)((unit - first) / x.units);
    x.first = first + (long long)x.head * x.units;
    return x;
}
__device__ __forceinline__ ChunkItem chunk_next(const ChunkArgs& a, const ChunkMap& m, ChunkItem x) {
    x.first += x.units;
    if (++x.head == a.kv_heads) {
        x.head = 0;
        if (++x.tile < m.tiles) x.units = (int)(m.unit_first[x.tile + 1] - m.unit_first[x.tile]);
    }
    return x;
}
__device__ __forceinline__ int chunk_slot_of(const ChunkArgs& a, const ChunkMap& m, int tile) {
    return chunk_owner(m.slot_first, a.slots, tile);
}
// First unit of CTA c's share.  Items of at most m.snap units are not cut: the border goes to
// their nearer end.
static __device__ __noinline__ long long chunk_border(const ChunkArgs& a, const ChunkMap& m, int c) {
    const long long u = c >= m.ctas ? m.units : m.units * c / m.ctas;
    if (u >= m.units || m.snap == 0) return u;
    const ChunkItem x = chunk_item(a, m, u);
    if (x.units > m.snap) return u;
    return u - x.first <= x.units / 2 ? x.first : x.first + x.units;
}
// The CTA in whose share a unit of an item above m.snap units lies (such items are cut at the plain borders)
__device__ __forceinline__ int chunk_cta_of(const ChunkMap& m, long long unit) {
    return (int)(((unit + 1) * m.ctas - 1) / m.units);
}

constexpr int CH_DESC = 8;  // {CTAs after this one, first packed row, rows, first row of the slot, key head, -, -, -}

cudaError_t launch_chunk_tc(const ChunkArgs& a, const CUtensorMap& map, int head_dim, int dtype, int ctas, cudaStream_t s);
cudaError_t launch_chunk_merge(const ChunkArgs& a, int head_dim, int tile_rows, int dtype, int ctas, cudaStream_t s);

}  // namespace mtp
