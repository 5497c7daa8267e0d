// chunk_plan.cu -- the plan of a chunk attention call (chunk.cuh): its tiles, every CTA's
// first item, and which items several CTAs share.  One CTA; prefix sums over the slots, over
// the tiles' units, then a thread per CTA of the kernel that follows.  What bounds it is
// latency: two scans and a few dependent loads.
#include "chunk.cuh"

namespace mtp {
namespace {

constexpr int PL_THREADS = 1024, PL_WARPS = PL_THREADS / 32;

// A slot in shared memory: its first row, new tokens (as far as they lie in the row buffers), length.
struct Slot {
    int row0, n, len;
};
__device__ __forceinline__ Slot load_slot(const ChunkArgs& a, int s) {
    Slot x;
    x.row0 = a.cu_rows[s];
    x.n = a.cu_rows[s + 1] - x.row0;
    x.len = max(0, min(a.kv_lens[s], a.bt_stride << a.page_shift));
    if (x.row0 < 0 || x.row0 > a.rows || x.n < 0) x.n = 0;
    x.n = min(x.n, a.rows - x.row0);
    return x;
}

template <int TR, int KT>
__device__ __forceinline__ ChunkTile make_tile(const ChunkArgs& a, int slot, const Slot& y, int t) {
    ChunkTile x;
    x.slot = slot;
    x.row0 = y.row0;
    x.p0 = t * TR;
    x.rows = min(y.n * a.group - x.p0, TR);
    x.base = y.len - y.n;
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

// Exclusive prefix sum of x over the block, and the total.
__device__ __forceinline__ uint32_t scan(uint32_t x, uint32_t* part, uint32_t& sum) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t y = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(FULL_MASK, y, o);
        if (lane >= o) y += u;
    }
    __syncthreads();  // `part` may still be read from an earlier call
    if (lane == 31) part[warp] = y;
    __syncthreads();
    const uint32_t mine = lane < PL_WARPS ? part[lane] : 0;
    sum = __reduce_add_sync(FULL_MASK, mine);
    return __reduce_add_sync(FULL_MASK, lane < warp ? mine : 0) + y - x;
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

// The stream in cost: an item costs its units and a.item_cost for its start and end, which come first.
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

// Shares and merges, in 32 bits where the cost times the CTAs fits (64-bit divisions were most of
// the plan's time).  CTA c's share begins at c / ctas of the cost; items of at most m.snap units
// are not cut: the border goes to their nearer end.
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
    const uint32_t extra = a.item_cost;
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

template <class U>
__device__ __forceinline__ void share_out(const ChunkArgs& a, const Map& m, U cost, U units, const ChunkTile* tiles,
                                          Border<U>* borders) {
    for (int c = threadIdx.x; c <= a.ctas; c += PL_THREADS) borders[c] = border<U>(a, m, cost, units, c);
    __syncthreads();
    for (int c = threadIdx.x; c < a.ctas; c += PL_THREADS) {
        const Border<U> x = borders[c], y = borders[c + 1];
        int4 start = make_int4(0, 0, 0, 0);
        int more = 0;
        int4* to = reinterpret_cast<int4*>(a.start + c);
        if (x.at < y.at) {
            start = make_int4(x.tile, x.head, x.k, (int)(y.unit - x.unit));
            const int4* from = reinterpret_cast<const int4*>(tiles + x.tile);
            to[1] = from[0];
            to[2] = from[1];
            to[3] = from[2];
            // the item that this share ends in, where it begins in the share and goes on, up to the CTA with its last unit
            if (y.k > 0 && (x.tile != y.tile || x.head != y.head || x.k == 0)) {
                more = 1;
                while (borders[c + 1 + more].at < y.item_end) ++more;
                const ChunkTile& t = tiles[y.tile];
                int* d = a.desc + c * CH_DESC;
                d[1] = t.p0;
                d[2] = t.rows;
                d[3] = t.row0;
                d[4] = y.head;
            }
        }
        to[0] = start;
        a.desc[c * CH_DESC] = more;
    }
}

// Shared memory: borders, the tiles where they are few, slots, first tile of every slot, first unit of every tile.
constexpr int PL_KEPT = 512;
__host__ __device__ inline size_t border_bytes(int ctas) { return ((size_t)(ctas + 1) * sizeof(Border<unsigned long long>) + 15) & ~(size_t)15; }
size_t plan_smem(const ChunkArgs& a) {
    return border_bytes(a.ctas) + (a.max_tiles <= PL_KEPT ? a.max_tiles * sizeof(ChunkTile) : 0) + (size_t)a.slots * sizeof(Slot) + (size_t)(a.slots + a.max_tiles + 2) * 4;
}

template <int TR, int KT>
__global__ void __launch_bounds__(PL_THREADS) chunk_plan_kernel(const __grid_constant__ ChunkArgs a) {
    extern __shared__ __align__(16) unsigned char pl_sm[];
    __shared__ uint32_t part[PL_WARPS];
    const bool keep = a.max_tiles <= PL_KEPT;
    ChunkTile* kept = reinterpret_cast<ChunkTile*>(pl_sm + border_bytes(a.ctas));
    Slot* slots = reinterpret_cast<Slot*>(kept + (keep ? a.max_tiles : 0));
    uint32_t* slot_first = reinterpret_cast<uint32_t*>(slots + a.slots);  // [slots + 1]
    uint32_t* unit_first = slot_first + a.slots + 1;                      // [tiles + 1]
    const int tid = threadIdx.x;
    pdl_launch_dependents();
    uint32_t base = 0, sum;  // (tiles: the kept rows of all slots lie in the buffers; a caller's wrong row starts: cut below)
    for (int s0 = 0; s0 < a.slots; s0 += PL_THREADS) {
        const int s = s0 + tid;
        uint32_t x = 0;
        if (s < a.slots) {
            const Slot y = load_slot(a, s);
            slots[s] = y;
            x = ((uint32_t)y.n * a.group + TR - 1) / TR;
        }
        x = scan(x, part, sum);
        if (s < a.slots) slot_first[s] = min(base + x, (uint32_t)a.max_tiles);
        base = min(base + sum, (uint32_t)a.max_tiles);
    }
    Map m;
    m.unit_first = unit_first;
    m.tiles = (int)base;
    if (tid == 0) slot_first[a.slots] = base;
    __syncthreads();
    base = 0;
    for (int j0 = 0; j0 < m.tiles; j0 += PL_THREADS) {
        const int j = j0 + tid;
        uint32_t x = 0;
        if (j < m.tiles) {
            const int s = owner(slot_first, a.slots, (uint32_t)j);
            const ChunkTile t = make_tile<TR, KT>(a, s, slots[s], j - (int)slot_first[s]);
            const int4* from = reinterpret_cast<const int4*>(&t);
            int4* to = reinterpret_cast<int4*>(a.tiles + j);
            to[0] = from[0];
            to[1] = from[1];
            to[2] = from[2];
            if (keep) kept[j] = t;
            x = t.units;
        }
        x = scan(x, part, sum);
        if (j < m.tiles) unit_first[j] = base + x;
        base += sum;
    }
    if (tid == 0) unit_first[m.tiles] = base;
    __syncthreads();
    const unsigned long long units = (unsigned long long)base * a.kv_heads;
    const unsigned long long cost = ((unsigned long long)base + (unsigned long long)m.tiles * a.item_cost) * a.kv_heads;
    const bool narrow = cost * a.ctas < 1ull << 32;
    m.ctas = (int)min((unsigned long long)a.ctas,
                      max(1ull, narrow ? (unsigned long long)(((uint32_t)units + a.min_units - 1) / a.min_units)
                                       : (units + a.min_units - 1) / a.min_units));
    m.snap = a.snap > 0 ? (int)min((unsigned long long)a.snap, narrow ? (uint32_t)units / m.ctas / 3 : units / m.ctas / 3) : 0;
    const ChunkTile* tiles = keep ? kept : a.tiles;
    if (narrow)
        share_out<uint32_t>(a, m, (uint32_t)cost, (uint32_t)units, tiles, reinterpret_cast<Border<uint32_t>*>(pl_sm));
    else
        share_out<unsigned long long>(a, m, cost, units, tiles, reinterpret_cast<Border<unsigned long long>*>(pl_sm));
}

template <int TR, int KT>
cudaError_t launch(const ChunkArgs& a, cudaStream_t s) {
    const size_t smem = plan_smem(a);
    const auto kern = chunk_plan_kernel<TR, KT>;
    const cudaError_t e = ensure_kernel_smem(reinterpret_cast<const void*>(kern), smem);
    return e == cudaSuccess ? launch_ex(kern, dim3(1), PL_THREADS, smem, false, s, a) : e;
}

}  // namespace

cudaError_t launch_chunk_plan(const ChunkArgs& a, int tile_rows, cudaStream_t s) {
    switch (tile_rows) {
        case 16: return launch<16, 64>(a, s);
        case 128: return launch<128, 128>(a, s);
        default: return launch<256, 128>(a, s);
    }
}

}  // namespace mtp
