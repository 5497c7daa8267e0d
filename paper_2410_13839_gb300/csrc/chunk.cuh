// chunk.cuh -- the work of a chunk attention call and how it is shared out, for
// both of its kernels (chunk_attention.cu, chunk_attention_tc.cu).
//
// The query heads that share a key head are rows of one product: row p of a slot and
// key head is token p / G, query head h G + p % G (G = heads per key head).  TR
// consecutive rows are a tile; with one key head it is an item.  An item's keys, from the
// first that one of its rows sees to the last, are cut into units of KT keys.  The units
// of all items, item after item, are one stream, of which CTA c of N takes the c-th N-th:
// ragged slots, few long ones or many short ones all give CTAs of equal work, at one
// prologue each.  In that sharing an item counts ITEM_COST units more than it has, for its start
// and end.  A plan kernel of one CTA writes the tiles, every CTA's first item and the merges into
// the workspace; under programmatic launch the kernel after it sets itself up meanwhile.  (Made
// by every CTA for itself, the plan of 25 prompts' tiles cost 85 us a call where the kernel's
// costs 66.)  A decoding step has one tile per slot: where its slots are at most FR_SLOTS, every CTA
// makes its own share's plan in shared memory, and the launch and the wait for it are saved (32
// slots of up to 2000 keys 36.4 us with the plan kernel, 33.1 without; 8 slots 14.2 and 11.0).
//
// An item that lies in one CTA's share is written by that CTA.  One that several share leaves
// (maximum, sum, unnormalised output) per row and CTA in the workspace, and a merge kernel
// after this one joins them by their maxima, in the CTAs' order: nothing depends on which CTA
// ends first.
#pragma once
#include "serving.cuh"

namespace mtp {

constexpr int CH_MAX_SLOTS = 4096, CH_MAX_PACKED = 1 << 21;
constexpr int CH_STEP = 64;  // keys of a step of the many-rows kernel
// An item's start and end, in units.  0, 1, 2, 3: 25 prompts 52.4, 43.4, 41.6, 42.3 us; a step of 32 slots 36.4, 34.8,
// 33.1, 32.6; windows of 1000 keys 104, 97, 97, 103.
constexpr int ITEM_COST = 2;

// A tile in the workspace: three 16-byte pieces.
struct ChunkTile {
    int slot, row0, p0, rows;  // the slot, its first row, packed rows [p0, p0 + rows)
    int base, lo, hi, units;   // position of the slot's first new token; keys [lo, hi) that some row sees (none: both 0); units
    int4 steps;                // steps of CH_STEP keys [x, y) of which the first 128 rows see a key, [z, w) the others
};
static_assert(sizeof(ChunkTile) == 48, "three pieces");

// Where a CTA's share begins: tile (a copy of it, for one look-up less), key head, unit of the item; units of the share.
struct ChunkStart {
    int tile, head, k, units;
    ChunkTile t;
};
static_assert(sizeof(ChunkStart) == 64, "four pieces");

// Tiles of 128 rows of a CTA of the many-rows kernel, and CTAs of an SM (they fill TMEM).  One tile of 64
// dims and two CTAs: bound by the softmax, they need no shared keys, and a tile's start and
// end lie behind the other CTA's work.  128 dims: two tiles, which share the copies of their keys
// and values (two CTAs' rings would not fit shared memory).
constexpr int chunk_tc_tiles(int head_dim) { return head_dim == 64 ? 1 : 2; }

struct ChunkArgs {
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    const int *block_table, *cu_rows, *kv_lens;
    long long q_stride, out_stride;
    int slots, rows, kv_heads, group, page_shift, bt_stride, n_pages;
    uint32_t group_inv;            // ceil(2^32 / group)
    int page_blocks, layer_block;  // (layer, K | V, head) blocks of a page; the layer's first
    int window, max_tiles, min_units, ctas;
    int snap;                      // items of at most so many units (and a third of a share) are not cut
    bool plan_here;                // few rows, few slots: every CTA makes its share itself
    bool q_vec, out_vec;           // rows 16-byte aligned
    bool residues;                 // the weights enter with their rounding residues
    bool q_tma;                    // many rows: Q's tiles are copied by a tensor map
    float scale_log2;              // scale * log2 e: scores in log2 units
    ChunkStart* start;             // [ctas]
    int* desc;                     // [ctas][CH_DESC]: merges
    ChunkTile* tiles;              // [max_tiles]
    float* part;                   // [ctas][2][TR][dim + 2]
    int* err;
};
constexpr int CH_DESC = 8;  // {CTAs after this one, first packed row, rows, first row of the slot, key head, -, -, -}

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

// A CTA's walk over the items of its share: the item, and its units [k0, k1) in the share.
struct PlannedTiles {  // the plan kernel's
    __device__ __forceinline__ ChunkTile operator()(const ChunkArgs& a, int tile) const {
        ChunkTile t;
        const int4* p = reinterpret_cast<const int4*>(a.tiles + tile);
        int4* to = reinterpret_cast<int4*>(&t);
        to[0] = p[0];
        to[1] = p[1];
        to[2] = p[2];
        return t;
    }
};
template <class TILES>
struct ChunkWalkOf {
    TILES tiles;
    int tile, head, k0, k1, left;  // left: units of the share from this item on
    ChunkTile t;
    __device__ __forceinline__ ChunkWalkOf(const ChunkStart& s, TILES from = TILES())
        : tiles(from), tile(s.tile), head(s.head), k0(s.k), left(s.units), t(s.t) {
        k1 = left > 0 ? min(t.units, k0 + left) : k0;
    }
    __device__ __forceinline__ void next(const ChunkArgs& a) {  // the item after this one (left 0: there is none)
        left -= k1 - k0;
        k0 = 0;
        if (left <= 0) return;
        if (++head == a.kv_heads) {
            head = 0;
            ++tile;
            t = tiles(a, tile);
        }
        k1 = min(t.units, left);
    }
    template <int KT>
    __device__ __forceinline__ int key0() const { return t.lo & ~(KT - 1); }  // first key of the item's first unit
    __device__ __forceinline__ bool begins() const { return k0 == 0; }
    __device__ __forceinline__ bool ends() const { return k1 == t.units; }
};
using ChunkWalk = ChunkWalkOf<PlannedTiles>;

// A slot: its first row, new tokens (as far as they lie in the row buffers), position of the first of them.
struct Slot {
    int row0, n, base;
};
// `cut` is set where rows that cu_rows gives the slot do not lie in the buffers (those that do keep their positions), and
// where the length of a slot with new tokens has no place in the table: such a slot has no key.
__device__ __forceinline__ Slot load_slot(const ChunkArgs& a, int s, bool& cut) {
    Slot x;
    x.row0 = a.cu_rows[s];
    const int end = a.cu_rows[s + 1], given = a.kv_lens[s];
    const bool placed = x.row0 >= 0 && end >= x.row0, held = given >= 0 && given <= a.bt_stride << a.page_shift;
    const int len = held ? given : 0;
    x.n = placed ? max(0, min(end, a.rows) - x.row0) : 0;
    // (fewer than CH_MAX_PACKED rows lie in the buffers: none of them reaches position 0 from further below)
    x.base = placed ? max(len - (end - x.row0), -CH_MAX_PACKED) : 0;
    cut |= !placed || end > a.rows || (x.n > 0 && !held);
    return x;
}

template <int TR, int KT>
__device__ __forceinline__ ChunkTile make_tile(const ChunkArgs& a, int slot, const Slot& y, int t) {
    ChunkTile x;
    x.slot = slot;
    x.row0 = y.row0;
    x.p0 = t * TR;
    x.rows = min(y.n * a.group - x.p0, TR);
    x.base = y.base;
    const int first = x.base + chunk_token(a, x.p0), last = x.base + chunk_token(a, x.p0 + x.rows - 1);  // positions
    x.hi = max(0, last + 1);
    x.lo = a.window > 0 ? min(x.hi, max(0, first - a.window + 1)) : 0;
    const int key0 = x.lo & ~(KT - 1);
    x.units = max(1, (x.hi - key0 + KT - 1) / KT);
    auto steps = [&](int p0, int rows) {  // of the keys that packed rows [p0, p0 + rows) see
        if (rows <= 0) return make_int2(0, 0);
        const int f = x.base + chunk_token(a, p0), l = x.base + chunk_token(a, p0 + rows - 1);
        const int hi = max(0, l + 1), lo = a.window > 0 ? max(0, f - a.window + 1) : 0;
        return hi <= lo ? make_int2(0, 0) : make_int2((lo - key0) / CH_STEP, (hi - key0 + CH_STEP - 1) / CH_STEP);
    };
    const int2 u = steps(x.p0, min(x.rows, 128)), v = steps(x.p0 + 128, x.rows - 128);
    x.steps = make_int4(u.x, u.y, v.x, v.y);
    return x;
}

// largest i in [0, n) with first[i] + i * extra <= x
template <class T>
__device__ __forceinline__ int owner(const T* first, int n, T x, T extra = 0) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] + mid * extra <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// The stream in cost: an item costs its units and ITEM_COST for its start and end, which come first.
struct Map {
    const uint32_t* unit_first;  // [tiles + 1]: first unit of every tile, counted for one key head
    int tiles, ctas, snap;
};
// A border between shares: a place in the cost, the item that begins or goes on there, the unit of the item that
// it stands before, the units before it.
template <class U>
struct Border {
    U at, unit, item_end;  // item_end: where the item ends in the cost
    int tile, head, k;
};

// CTA c's share begins at c / ctas of the cost; items of at most m.snap units are not cut: the border
// goes to their nearer end.  In 32 bits where the cost times the CTAs fits (64-bit divisions were most of the plan's time).
template <class U>
__device__ __forceinline__ Border<U> border(const ChunkArgs& a, const Map& m, U cost, U units, int c) {
    Border<U> x;
    x.at = x.item_end = cost;
    x.unit = units;
    x.tile = m.tiles;
    x.head = x.k = 0;
    if (c >= m.ctas) return x;
    const U u = cost * (U)c / (U)m.ctas;
    if (u >= cost) return x;
    constexpr uint32_t extra = ITEM_COST;
    x.tile = owner(m.unit_first, m.tiles, (uint32_t)(u / (U)a.kv_heads), extra);
    const uint32_t unit0 = m.unit_first[x.tile], n = m.unit_first[x.tile + 1] - unit0;
    const U first = ((U)unit0 + (U)x.tile * extra) * (U)a.kv_heads, item = (U)n + extra;
    x.head = (int)((uint32_t)(u - first) / (uint32_t)item);  // (an item's cost and heads: below 2^32 together)
    x.at = first + (U)x.head * item;
    x.unit = (U)unit0 * (U)a.kv_heads + (U)x.head * (U)n;
    x.item_end = x.at + item;
    const uint32_t in = (uint32_t)(u - x.at);
    if (n <= (uint32_t)m.snap) {
        if (in > (n + extra) / 2) {  // the next item's start
            x.at += item;
            x.unit += n;
            if (++x.head == a.kv_heads) {
                x.head = 0;
                ++x.tile;
            }
            const uint32_t next = x.tile < m.tiles ? m.unit_first[x.tile + 1] - m.unit_first[x.tile] : 0;
            x.item_end = x.at + (U)next + extra;
        }
    } else if (in > extra) {
        x.k = (int)(in - extra);
        x.unit += (U)x.k;
        x.at = u;
    }
    return x;
}

// CTAs after c whose shares begin in the item that x cuts: floor(cost * i / ctas) < item_end
template <class U>
__device__ __forceinline__ int shares_after(const Border<U>& x, U cost, int ctas, int c) {
    return (int)((x.item_end * (U)ctas - 1) / cost) - c;
}

cudaError_t launch_chunk_plan(const ChunkArgs& a, int tile_rows, cudaStream_t s);  // 16; 128, 256: many rows
cudaError_t launch_chunk_tc(const ChunkArgs& a, const CUtensorMap& map, const CUtensorMap& q_map, int head_dim, int dtype,
                            cudaStream_t s);

}  // namespace mtp
