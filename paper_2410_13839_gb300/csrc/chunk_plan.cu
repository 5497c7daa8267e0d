// chunk_plan.cu -- the plan of a chunk attention call (chunk.cuh): its tiles, every CTA's
// first item, and which items several CTAs share.  One CTA; prefix sums over the slots, over
// the tiles' units, then a thread per border between shares.  What bounds it is latency: two
// scans and a few dependent loads, about 3 us with 32 slots.
#include "chunk.cuh"

namespace mtp {
namespace {

constexpr int PL_THREADS = 512, PL_WARPS = PL_THREADS / 32;

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

template <class U>
__device__ __forceinline__ void share_out(const ChunkArgs& a, const Map& m, U cost, U units, Border<U>* borders) {
    for (int c = threadIdx.x; c <= a.ctas; c += PL_THREADS) borders[c] = border<U>(a, m, cost, units, c);
    __syncthreads();
    for (int c = threadIdx.x; c < a.ctas; c += PL_THREADS) {
        const Border<U> x = borders[c], y = borders[c + 1];
        int4 start = make_int4(0, 0, 0, 0);
        int more = 0;
        int4* to = reinterpret_cast<int4*>(a.start + c);
        if (x.at < y.at) {
            start = make_int4(x.tile, x.head, x.k, (int)(y.unit - x.unit));
            const int4* from = reinterpret_cast<const int4*>(a.tiles + x.tile);
            to[1] = from[0];
            to[2] = from[1];
            to[3] = from[2];
            // the item that this share ends in, where it begins in the share and goes on, up to the CTA with its last unit
            if (y.k > 0 && (x.tile != y.tile || x.head != y.head || x.k == 0)) {
                more = shares_after(y, cost, m.ctas, c);
                const ChunkTile& t = a.tiles[y.tile];
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

// Shared memory: borders, slots, first tile of every slot, first unit of every tile.
__host__ __device__ inline size_t border_bytes(int ctas) { return ((size_t)(ctas + 1) * sizeof(Border<unsigned long long>) + 15) & ~(size_t)15; }
size_t plan_smem(const ChunkArgs& a) {
    return border_bytes(a.ctas) + (size_t)a.slots * sizeof(Slot) + (size_t)(a.slots + a.max_tiles + 2) * 4;
}

template <int TR, int KT>
__global__ void __launch_bounds__(PL_THREADS) chunk_plan_kernel(const __grid_constant__ ChunkArgs a) {
    extern __shared__ __align__(16) unsigned char pl_sm[];
    __shared__ uint32_t part[PL_WARPS];
    Slot* slots = reinterpret_cast<Slot*>(pl_sm + border_bytes(a.ctas));
    uint32_t* slot_first = reinterpret_cast<uint32_t*>(slots + a.slots);  // [slots + 1]
    uint32_t* unit_first = slot_first + a.slots + 1;                      // [tiles + 1]
    const int tid = threadIdx.x;
    pdl_launch_dependents();
    pdl_wait();
    uint32_t base = 0, sum;  // (more tiles than the workspace has, by a max_new too small or slots that overlap, are left out)
    bool cut = false;
    for (int s0 = 0; s0 < a.slots; s0 += PL_THREADS) {
        const int s = s0 + tid;
        uint32_t x = 0;
        if (s < a.slots) {
            const Slot y = load_slot(a, s, cut);
            slots[s] = y;
            x = ((uint32_t)y.n * a.group + TR - 1) / TR;
        }
        x = scan(x, part, sum);
        if (s < a.slots) slot_first[s] = min(base + x, (uint32_t)a.max_tiles);
        cut |= base + sum > (uint32_t)a.max_tiles;
        base = min(base + sum, (uint32_t)a.max_tiles);
    }
    if (cut && a.err) atomicOr(a.err, ERR_BOUNDS);
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
            x = t.units;
        }
        x = scan(x, part, sum);
        if (j < m.tiles) unit_first[j] = base + x;
        base += sum;
    }
    if (tid == 0) unit_first[m.tiles] = base;
    __syncthreads();
    const unsigned long long units = (unsigned long long)base * a.kv_heads;
    const unsigned long long cost = ((unsigned long long)base + (unsigned long long)m.tiles * ITEM_COST) * a.kv_heads;
    const bool narrow = cost * a.ctas < 1ull << 32;
    m.ctas = (int)min((unsigned long long)a.ctas,
                      max(1ull, narrow ? (unsigned long long)(((uint32_t)units + a.min_units - 1) / a.min_units)
                                       : (units + a.min_units - 1) / a.min_units));
    m.snap = a.snap > 0 ? (int)min((unsigned long long)a.snap, narrow ? (uint32_t)units / m.ctas / 3 : units / m.ctas / 3) : 0;
    if (narrow)
        share_out<uint32_t>(a, m, (uint32_t)cost, (uint32_t)units, reinterpret_cast<Border<uint32_t>*>(pl_sm));
    else
        share_out<unsigned long long>(a, m, cost, units, reinterpret_cast<Border<unsigned long long>*>(pl_sm));
}

template <int TR, int KT>
cudaError_t launch(const ChunkArgs& a, cudaStream_t s) {
    const size_t smem = plan_smem(a);
    const auto kern = chunk_plan_kernel<TR, KT>;
    const cudaError_t e = ensure_kernel_smem(reinterpret_cast<const void*>(kern), smem);
    return e == cudaSuccess ? launch_ex(kern, dim3(1), PL_THREADS, smem, s, 1, a) : e;
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
