// chunk_plan.cu -- the plan of a chunk attention call (chunk.cuh): its tiles, every CTA's
// first item, and which items several CTAs share.  One CTA; prefix sums over the slots, over
// the tiles' units, then a thread per CTA of the kernel that follows.  What bounds it is
// latency: two scans and a few dependent loads.
#include "chunk.cuh"

namespace mtp {
namespace {

constexpr int PL_THREADS = 1024, PL_WARPS = PL_THREADS / 32;

// rows of slot s, as far as they lie in the row buffers
__device__ __forceinline__ void slot_rows(const ChunkArgs& a, int s, int& row0, int& n) {
    row0 = a.cu_rows[s];
    n = a.cu_rows[s + 1] - row0;
    if (row0 < 0 || row0 > a.rows || n < 0) n = 0;
    n = min(n, a.rows - row0);
}

template <int TR, int KT>
__device__ __forceinline__ ChunkTile make_tile(const ChunkArgs& a, int slot, int t) {
    ChunkTile x;
    int n;
    x.slot = slot;
    slot_rows(a, slot, x.row0, n);
    const int len = max(0, min(a.kv_lens[slot], a.bt_stride << a.page_shift));
    x.p0 = t * TR;
    x.rows = min(n * a.group - x.p0, TR);
    x.base = len - n;
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

template <class T>
__device__ __forceinline__ int owner(const T* first, int n, T x) {  // largest i in [0, n) with first[i] <= x
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

struct Map {
    const uint32_t* unit_first;  // [tiles + 1]: first unit of every tile, counted for one key head
    int tiles, ctas, snap;
    long long units;             // of all key heads
};
struct Item {
    int tile, head, units;
    long long first;  // its first unit
};
__device__ __forceinline__ Item item_of(const ChunkArgs& a, const Map& m, long long unit) {
    Item x;
    x.tile = owner(m.unit_first, m.tiles, (uint32_t)(unit / a.kv_heads));
    const long long first = (long long)m.unit_first[x.tile] * a.kv_heads;
    x.units = (int)(m.unit_first[x.tile + 1] - m.unit_first[x.tile]);
    x.head = (int)((uint32_t)(unit - first) / (uint32_t)x.units);  // (an item's units and heads: below 2^32 together)
    x.first = first + (long long)x.head * x.units;
    return x;
}
// First unit of CTA c's share.  Items of at most m.snap units are not cut: the border goes to
// their nearer end.
__device__ __forceinline__ long long border(const ChunkArgs& a, const Map& m, int c) {
    const long long u = c >= m.ctas ? m.units : m.units * c / m.ctas;
    if (u >= m.units || m.snap == 0) return u;
    const Item x = item_of(a, m, u);
    if (x.units > m.snap) return u;
    return u - x.first <= x.units / 2 ? x.first : x.first + x.units;
}

template <int TR, int KT>
__global__ void __launch_bounds__(PL_THREADS) chunk_plan_kernel(const __grid_constant__ ChunkArgs a) {
    extern __shared__ int pl_sm[];
    __shared__ long long part[PL_WARPS][2];
    int* slot_first = pl_sm;                                              // [slots + 1]: first tile of every slot
    uint32_t* unit_first = reinterpret_cast<uint32_t*>(pl_sm + a.slots + 1);  // [tiles + 1]
    const int tid = threadIdx.x;
    pdl_launch_dependents();
    long long base = 0, unused = 0, sum, none;
    for (int s0 = 0; s0 < a.slots; s0 += PL_THREADS) {
        const int s = s0 + tid;
        long long x = 0;
        if (s < a.slots) {
            int row0, n;
            slot_rows(a, s, row0, n);
            x = ((long long)n * a.group + TR - 1) / TR;
        }
        block_scan2<PL_WARPS>(x, unused, part, sum, none);
        if (s < a.slots) slot_first[s] = (int)min(base + x, (long long)a.max_tiles);
        base += sum;
    }
    Map m;
    m.unit_first = unit_first;
    m.tiles = (int)min(base, (long long)a.max_tiles);
    if (tid == 0) slot_first[a.slots] = m.tiles;
    __syncthreads();
    base = 0;
    for (int j0 = 0; j0 < m.tiles; j0 += PL_THREADS) {
        const int j = j0 + tid;
        long long x = 0;
        if (j < m.tiles) {
            const int s = owner(slot_first, a.slots, j);
            const ChunkTile t = make_tile<TR, KT>(a, s, j - slot_first[s]);
            const int4* from = reinterpret_cast<const int4*>(&t);
            int4* to = reinterpret_cast<int4*>(a.tiles + j);
            to[0] = from[0];
            to[1] = from[1];
            to[2] = from[2];
            x = t.units;
        }
        block_scan2<PL_WARPS>(x, unused, part, sum, none);
        if (j < m.tiles) unit_first[j] = (uint32_t)(base + x);
        base += sum;
    }
    if (tid == 0) unit_first[m.tiles] = (uint32_t)base;
    __syncthreads();
    m.units = base * a.kv_heads;
    m.ctas = (int)min((long long)a.ctas, max(1ll, (m.units + a.min_units - 1) / a.min_units));
    m.snap = a.snap ? (int)min(m.units / m.ctas / a.snap, 1ll << 30) : 0;
    for (int c = tid; c < a.ctas; c += PL_THREADS) {
        const long long u0 = border(a, m, c), u1 = border(a, m, c + 1);
        int4 start = make_int4(0, 0, 0, 0);
        int more = 0;
        if (u0 < u1) {
            const Item x = item_of(a, m, u0);
            start = make_int4(x.tile, x.head, (int)(u0 - x.first), (int)(u1 - u0));
            if (u1 < m.units) {
                const Item y = item_of(a, m, u1);
                if (y.first < u1 && y.first >= u0) {  // begins here and goes on: up to the CTA with its last unit
                    const long long last = y.first + y.units - 1;
                    more = (int)(((last + 1) * m.ctas - 1) / m.units) - c;
                    int* d = a.desc + c * CH_DESC;
                    const ChunkTile& t = a.tiles[y.tile];
                    d[1] = t.p0;
                    d[2] = t.rows;
                    d[3] = t.row0;
                    d[4] = y.head;
                }
            }
        }
        a.start[c] = start;
        a.desc[c * CH_DESC] = more;
    }
}

template <int TR, int KT>
cudaError_t launch(const ChunkArgs& a, cudaStream_t s) {
    const size_t smem = (size_t)(a.slots + a.max_tiles + 2) * 4;
    const auto kern = chunk_plan_kernel<TR, KT>;
    const cudaError_t e = ensure_kernel_smem(reinterpret_cast<const void*>(kern), smem);
    return e == cudaSuccess ? launch_ex(kern, dim3(1), PL_THREADS, smem, false, s, a) : e;
}

}  // namespace

cudaError_t launch_chunk_plan(const ChunkArgs& a, int tile_rows, cudaStream_t s) {
    return tile_rows == 16 ? launch<16, 64>(a, s) : tile_rows == 32 ? launch<32, 64>(a, s) : launch<256, 128>(a, s);
}

}  // namespace mtp
