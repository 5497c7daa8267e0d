// chunk_attention.cu -- attention of a chunk of new tokens per slot over the paged
// cache (mtp_chunk_attention): its entry point, the kernel of few rows per slot and key
// head (decoding steps, drafts), and the merge of shared items.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = 2^(s_ij - m_i),  s_ij = scale log2(e) q_i . k_j,
//   lse_i = ln 2 (m_i + log2 sum_j p_ij),  j over the keys that token i sees,
//
// in one pass over the keys with a running maximum m_i (fp32, as the sums and outputs).
//
// Few rows: the keys are read once and used by few rows, so memory bounds it.  A CTA's
// share of the unit stream (chunk.cuh) runs through a ring of stages of 64 keys; the fifth
// warp fills them, a lane per page piece, with TMA copies that lay the rows out in the
// 128-byte swizzle that ldmatrix reads without bank conflicts.  Each of the four other
// warps takes 16 of a stage's keys: S = Q K^T and O += P V by mma.sync (16 rows of a tile
// as M), with a maximum, sum and output of its own, which the four join at the item's end.
// From 17 rows on the tensor cores' 128-row tiles are used, mostly empty (chunk_attention_tc.cu):
// 16 rows on 8 contexts of 4,000 to 30,000 keys, 128 dims fp16, take 79.7 us here and 92 there, on
// 32 of up to 2000 keys, 64 dims bf16, 12.9 and 21.9; 32 rows, in tiles of 32 rows made as
// these are, took 172 and 24.8, there 93.6 and 22.3, on 128 contexts 62 and 52.
//
// A decoding step of 32 slots (180 to 2000 keys, 16 heads of 64, 147 MB) takes 33 us a call, of
// which the memory's part is 21.6 us: the share's plan, the ring's start, an item's joining
// and the merge are the rest, 2 to 3 us each.  4 drafts of 8 slots of 4,000 to 30,000 keys, 8 key
// heads of 128 dims (480 MB): 79.7 us, 89 % of 6.8 TB/s.
//
// Q enters as it is (16 bits).  P enters as a pair hi + lo of the type, its rounding
// residue with it: a bound memory leaves the second product free, and the outputs then
// err by their own rounding alone (P rounded once would add as much again).
#include <algorithm>

#include "chunk.cuh"
#include "frag.cuh"

namespace mtp {

int tc_encode_cache(CUtensorMap* map, const void* pool, int dtype, int head_dim, int page_size, uint64_t blocks,
                    int box_rows);
int tc_encode_queries(CUtensorMap* map, const void* q, int dtype, int head_dim, int heads, uint64_t rows, uint64_t stride,
                      int group);

namespace {

constexpr int FR_KEYS = 64, FR_WARPS = 5, FR_THREADS = FR_WARPS * 32, FR_CONSUMERS = 128;
// Fewest units of a CTA.  Few rows, 2, 4, 8: 2 slots of up to 2000 keys 8.6, 10.2, 13.9 us, one of 32,000 keys and 2 key heads, whose
// merge grows, 19.3, 16.6, 15.9; many rows, 1, 2, 4: 4 prompts 18.3, 19.4, 22.3.
constexpr int FR_MIN_UNITS = 4, CT_MIN_UNITS = 1;
// Items of many rows of at most so many units are not cut: a cut costs a tile's parts and their merge, about two units'
// time.  All cut, 6, 12, 24: windows of 1000 keys 105, 105, 97, 97 us, 25 prompts of 128 dims 72.6, 67.9, 68.1, 67.7; items of
// many slots are better cut: 128 slots of 32 rows, 128 dims, 77.7, 79.5, 84.0, 84.0, 64 dims 51.4, 52.2, 52.2, 52.2.  (Up to a third
// of a share, however long: chunks of thousands of tokens 486 us instead of 447.)
constexpr int CT_SNAP = 12;
constexpr int FR_ROWS = 16, CT_UNIT_KEYS = 128;  // a tile of few rows
constexpr int FR_SLOTS = 128;                   // slots whose plan every CTA makes for itself
constexpr int RESIDUE_ROWS = 32;  // rows of a slot and key head up to which the weights' residues are kept
constexpr float LN2 = 0.69314718055994531f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void tma_cache(void* dst, const CUtensorMap* map, int x, int row, int block, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            smem_addr(dst)),
        "l"(map), "r"(x), "r"(row), "r"(block), "r"(smem_addr(bar))
        : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, %0;" ::"n"(FR_CONSUMERS) : "memory"); }

template <class T>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<Bf16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<F16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <class T>
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = T::pack(x, y);
    lo = T::pack(x - T::to_float((uint16_t)hi), y - T::to_float((uint16_t)(hi >> 16)));
}

// Shared memory of the few-rows kernel, from a 1024-byte boundary: ring stages (K then V, each
// HD / 64 tiles of 64 rows of 128 bytes), Q (HD / 64 tiles of TR rows), a join buffer of TR x HD
// floats, per-warp maxima and sums.
template <int HD>
struct FrLayout {
    static constexpr int TR = FR_ROWS;
    static constexpr int STAGES = HD == 64 ? 4 : 3;
    static constexpr uint32_t TILE = FR_KEYS * 128, KV = TILE * (HD / 64), STAGE = 2 * KV;
    static constexpr uint32_t Q = STAGES * STAGE, JOIN = Q + TR * HD * 2, ML = JOIN + TR * HD * 4;
    static constexpr size_t BYTES = 1024 + ML + 2 * 4 * TR * 4;
};

// Few slots: a tile each (those without new tokens have none), with the first unit of each, in shared memory.
struct FewSlots {
    Slot slot[FR_SLOTS];
    int number[FR_SLOTS];
    uint32_t first[FR_SLOTS + 1], warp_units[4], warp_tiles[4];
    Border<uint32_t> border[2];
};
struct FewTiles {
    const FewSlots* f;
    __device__ __forceinline__ ChunkTile operator()(const ChunkArgs& a, int tile) const {
        return a.plan_here ? make_tile<FR_ROWS, FR_KEYS>(a, f->number[tile], f->slot[tile], 0) : PlannedTiles()(a, tile);
    }
};
// The plan's work for one CTA: where its share begins, and its merge.  The whole CTA calls it.
__device__ __forceinline__ ChunkStart plan_share(const ChunkArgs& a, FewSlots& f) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    Slot y{0, 0, 0};
    uint32_t units = 0;
    bool cut = false;
    if (tid < a.slots) {
        y = load_slot(a, tid, cut);
        if (y.n > 0) units = make_tile<FR_ROWS, FR_KEYS>(a, tid, y, 0).units;
        cut |= y.n * a.group > FR_ROWS;  // rows past the slot's tile: max_new was too small
    }
    if (cut && cta == 0 && a.err) atomicOr(a.err, ERR_BOUNDS);
    const unsigned live = __ballot_sync(FULL_MASK, units > 0);
    uint32_t x = units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(FULL_MASK, x, o);
        if (lane >= o) x += u;
    }
    if (lane == 31 && warp < 4) {
        f.warp_units[warp] = x;
        f.warp_tiles[warp] = __popc(live);
    }
    __syncthreads();
    uint32_t all = 0, tiles = 0, j = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w == warp) {
            x += all;
            j = tiles;
        }
        all += f.warp_units[w];
        tiles += f.warp_tiles[w];
    }
    if (units > 0) {
        j += __popc(live & ((1u << lane) - 1));
        f.slot[j] = y;
        f.number[j] = tid;
        f.first[j] = x - units;
    }
    if (tid == 0) f.first[tiles] = all;
    __syncthreads();
    Map m;
    m.unit_first = f.first;
    m.tiles = (int)tiles;
    m.snap = 0;
    const uint32_t sum = all * a.kv_heads, cost = sum + tiles * ITEM_COST * a.kv_heads;
    m.ctas = min(a.ctas, max(1, (int)((sum + a.min_units - 1) / a.min_units)));
    if (lane == 0 && warp < 2) f.border[warp] = border<uint32_t>(a, m, cost, sum, cta + warp);
    __syncthreads();
    const Border<uint32_t> at = f.border[0], end = f.border[1];
    ChunkStart s;
    s.tile = s.head = s.k = s.units = 0;
    int more = 0;
    if (at.at < end.at) {
        s.tile = at.tile;
        s.head = at.head;
        s.k = at.k;
        s.units = (int)(end.unit - at.unit);
        s.t = make_tile<FR_ROWS, FR_KEYS>(a, f.number[at.tile], f.slot[at.tile], 0);
        if (tid == 0 && end.k > 0 && (at.tile != end.tile || at.head != end.head || at.k == 0)) {
            more = shares_after(end, cost, m.ctas, cta);
            const Slot& z = f.slot[end.tile];
            int* d = a.desc + cta * CH_DESC;
            d[1] = 0;
            d[2] = min(z.n * a.group, FR_ROWS);
            d[3] = z.row0;
            d[4] = end.head;
        }
    }
    if (tid == 0) a.desc[cta * CH_DESC] = more;
    return s;
}

template <class T, int HD>
__global__ void __launch_bounds__(FR_THREADS, HD == 64 ? 3 : 2)
    chunk_rows_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ CUtensorMap map) {
    using L = FrLayout<HD>;
    constexpr int TR = L::TR, ST = L::STAGES;
    extern __shared__ unsigned char fr_raw[];
    __shared__ uint64_t full[ST], empty[ST];
    __shared__ FewSlots few;
    unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(fr_raw) + 1023) & ~(uintptr_t)1023);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    if (tid == 0) {
        for (int i = 0; i < ST; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 4);
        }
        fence_barrier_init();
    }
    __syncthreads();
    pdl_launch_dependents();
    pdl_wait();  // the plan, or the kernels before this call
    const ChunkStart start = a.plan_here ? plan_share(a, few) : a.start[cta];
    const int units = start.units;
    if (units == 0) return;

    if (warp == 4) {  // ---- the ring's filler ----
        const int P = 1 << a.page_shift, box = min(P, FR_KEYS), per = FR_KEYS / box;
        // this lane's piece of a stage: rows [sub * box, + box) of half `half` of K (0) or V (1)
        const int sub = lane % per, half = lane / per % (HD / 64), kv = lane / per / (HD / 64);
        const bool mine = kv < 2;
        unsigned char* ring = sm + kv * L::KV + half * L::TILE + sub * box * 128;
        ChunkWalkOf<FewTiles> w(start, FewTiles{&few});
        int k = w.k0, issued = 0, base = 0, pages = 0, ahead = 0;
        bool ok = true;
        // pages [base, base + 32) of the slot, one per lane, and the 32 after them
        auto lookup = [&](int first) {
            return first + lane < a.bt_stride ? *(a.block_table + (size_t)w.t.slot * a.bt_stride + first + lane) : -1;
        };
        auto enter = [&]() {
            base = (w.key0<FR_KEYS>() + k * FR_KEYS) >> a.page_shift & ~31;
            pages = lookup(base);
            ahead = lookup(base + 32);
        };
        enter();
        for (; issued < units; ++issued) {
            const int st = issued % ST, key = w.key0<FR_KEYS>() + k * FR_KEYS + sub * box, index = key >> a.page_shift;
            if (index - base >= 32) {  // (the same in all lanes: a unit's pages lie in one aligned group)
                base += 32;
                pages = ahead;
                ahead = lookup(base + 32);
            }
            int page = __shfl_sync(FULL_MASK, pages, (index - base) & 31);
            page = page >= 0 && page < a.n_pages ? page : -1;  // -1: outside the pool, zeros
            const int block = page < 0 ? -1 : page * a.page_blocks + a.layer_block + kv * a.kv_heads + w.head;
            const bool wanted = mine && key < w.t.hi && key + box > w.t.lo;  // some row sees a key of the piece
            const unsigned have = __ballot_sync(FULL_MASK, wanted);
            if (issued >= ST) {
                ok = __all_sync(FULL_MASK, lane != 0 || chunk_wait(&empty[st], issued / ST - 1, a.err));
                if (!ok) break;
            }
            if (lane == 0) mbar_arrive_expect_tx(&full[st], __popc(have) * box * 128);
            __syncwarp();
            if (wanted) tma_cache(ring + st * L::STAGE, &map, half * 64, key & (P - 1), block, &full[st]);
            if (++k == w.k1 && issued + 1 < units) {
                w.next(a);
                k = 0;
                enter();
            }
        }
        // after a failed wait: what is in flight lands before the CTA leaves
        if (!ok && lane == 0)
            for (int i = max(0, issued - ST); i < issued; ++i) chunk_wait(&full[i % ST], i / ST, nullptr);
        return;
    }

    // ---- the rows ----
    const int r0 = lane >> 2, c0 = (lane & 3) * 2;  // this lane's rows r0, r0 + 8 of 16, columns c0, c0 + 1 of 8
    const uint32_t q_base = smem_addr(sm + L::Q);
    float* join = reinterpret_cast<float*>(sm + L::JOIN);
    float* ml = reinterpret_cast<float*>(sm + L::ML);  // [4 warps][TR] maxima, then sums
    int stage = 0;
    bool alive = true;
    ChunkWalkOf<FewTiles> w(start, FewTiles{&few});
    for (; w.left > 0; w.next(a)) {
        const ChunkTile& t = w.t;
        const int key_first = w.key0<FR_KEYS>();
        const bool begins = w.begins(), ends = w.ends();
        // Q: 16 bytes a thread and step, rows past the tile zero
        for (int i = tid; i < TR * (HD / 8); i += FR_CONSUMERS) {
            const int r = i / (HD / 8), c = i % (HD / 8), p = t.p0 + r;
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (r < t.rows) {
                const int token = chunk_token(a, p);
                const uint16_t* src = a.q + (t.row0 + token) * a.q_stride + (w.head * a.group + p - token * a.group) * HD + c * 8;
                if (a.q_vec) {
                    v = *reinterpret_cast<const uint4*>(src);
                } else {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = (uint32_t)*(src + 2 * e) | (uint32_t)*(src + 2 * e + 1) << 16;
                    v = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            *reinterpret_cast<uint4*>(sm + L::Q + (c >> 3) * (TR * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v;
        }
        consumer_sync();
        float o[HD / 8][4], mx[2], sum[2];
        int pos[2];  // the rows' positions
#pragma unroll
        for (int d = 0; d < HD / 8; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[d][e] = 0.f;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            mx[e] = -INFINITY;
            sum[e] = 0.f;
            const int r = r0 + e * 8;
            pos[e] = r < t.rows ? t.base + chunk_token(a, t.p0 + r) : -1;
        }
        const int pos_first = t.base + chunk_token(a, t.p0), pos_last = t.hi - 1;
        for (int k = w.k0; k < w.k1; ++k) {
            const int st = stage % ST;
            if (alive) alive = __all_sync(FULL_MASK, lane != 0 || chunk_wait(&full[st], stage / ST, a.err));
            const int key0 = key_first + k * FR_KEYS + warp * 16;  // this warp's keys
            if (alive && key0 < t.hi && key0 + 16 > t.lo) {
                unsigned char* kb = sm + st * L::STAGE;
                // a unit that every row sees in full needs no mask; its keys are all copied
                const bool inner = key0 + 15 <= pos_first && (a.window <= 0 || key0 > pos_last - a.window) && t.rows == TR;
                const bool edge = key0 + 16 > t.hi || key0 < t.lo;  // keys that no row sees: their values may be anything
                if (edge) {
                    const int r = lane >> 1, key = key0 + r;
                    if (key >= t.hi || key < t.lo)
                        for (int c = lane & 1; c < HD / 8; c += 2)
                            *reinterpret_cast<uint4*>(kb + L::KV + (c >> 3) * L::TILE + (warp * 16 + r) * 128 + (c & 7) * 16) =
                                make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async();  // (the stage is copied into again)
                    __syncwarp();
                }
                const uint32_t kr = smem_addr(kb), vr = kr + L::KV;
                float s[2][4];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[j][e] = 0.f;
#pragma unroll
                for (int d = 0; d < HD / 16; ++d) {
                    uint32_t kf[4];
                    const int key = warp * 16 + ((lane >> 4) << 3) + (lane & 7), c = 2 * d + ((lane >> 3) & 1);
                    frag::ldsm_x4(kf, kr + (c >> 3) * L::TILE + key * 128 + (((c & 7) ^ (key & 7)) << 4));
                    uint32_t qf[4];
                    const int row = lane & 15, cq = 2 * d + (lane >> 4);
                    frag::ldsm_x4(qf, q_base + (cq >> 3) * (TR * 128) + row * 128 + (((cq & 7) ^ (row & 7)) << 4));
                    mma16<T>(s[0], qf, kf[0], kf[1]);
                    mma16<T>(s[1], qf, kf[2], kf[3]);
                }
                uint32_t hi[4], lo[4];
                if (!inner) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = key0 + j * 8 + c0 + (e & 1), p = pos[e >> 1];
                            if (key > p || (a.window > 0 && key <= p - a.window)) s[j][e] = -INFINITY;
                        }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = fmaxf(fmaxf(s[0][2 * e], s[0][2 * e + 1]), fmaxf(s[1][2 * e], s[1][2 * e + 1]));
                    top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(FULL_MASK, top, 2));
                    const float now = fmaxf(mx[e], top * a.scale_log2);
                    if (__any_sync(FULL_MASK, now > mx[e])) {
                        const float f = mx[e] == -INFINITY ? 0.f : ex2(mx[e] - now);
                        sum[e] *= f;
#pragma unroll
                        for (int d = 0; d < HD / 8; ++d) {
                            o[d][2 * e] *= f;
                            o[d][2 * e + 1] *= f;
                        }
                        mx[e] = now;
                    }
                    const float ref = now == -INFINITY ? 0.f : now;  // a row that has seen no key: every weight 0
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float x = ex2(fmaf(s[j][2 * e], a.scale_log2, -ref)),
                                    y = ex2(fmaf(s[j][2 * e + 1], a.scale_log2, -ref));
                        sum[e] += x + y;
                        split2<T>(x, y, hi[2 * j + e], lo[2 * j + e]);
                    }
                }
#pragma unroll
                for (int d = 0; d < HD / 16; ++d) {
                    uint32_t vf[4];
                    const int key = warp * 16 + (lane & 15), c = 2 * d + (lane >> 4);
                    frag::ldsm_x4_t(vf, vr + (c >> 3) * L::TILE + key * 128 + (((c & 7) ^ (key & 7)) << 4));
                    mma16<T>(o[2 * d], hi, vf[0], vf[1]);
                    mma16<T>(o[2 * d + 1], hi, vf[2], vf[3]);
                    mma16<T>(o[2 * d], lo, vf[0], vf[1]);
                    mma16<T>(o[2 * d + 1], lo, vf[2], vf[3]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[st]);
            ++stage;
        }
        // ---- the four warps' maxima, sums and outputs as one ----
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            sum[e] += __shfl_xor_sync(FULL_MASK, sum[e], 1);
            sum[e] += __shfl_xor_sync(FULL_MASK, sum[e], 2);
            if ((lane & 3) == 0) {
                const int r = r0 + e * 8;
                ml[warp * TR + r] = mx[e];
                ml[(4 + warp) * TR + r] = sum[e];
            }
        }
        consumer_sync();
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = r0 + e * 8;
            float top = -INFINITY, all = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w * TR + r]);
            const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < 4; ++w) all = fmaf(ml[(4 + w) * TR + r], ex2(ml[w * TR + r] - ref), all);
            const float f = ex2(mx[e] - ref);
#pragma unroll
            for (int d = 0; d < HD / 8; ++d) {
                o[d][2 * e] *= f;
                o[d][2 * e + 1] *= f;
            }
            mx[e] = top;
            sum[e] = all;
        }
#pragma unroll
        for (int w = 3; w >= 0; --w) {  // warp 3 leaves its outputs, 2 and 1 add theirs, 0 takes the sum
            if (warp == w) {
#pragma unroll
                for (int d = 0; d < HD / 8; ++d) {
                    float4* at = reinterpret_cast<float4*>(join) + d * 32 + lane;
                    float4 v = make_float4(o[d][0], o[d][1], o[d][2], o[d][3]);
                    if (w < 3) {
                        const float4 x = *at;
                        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
                    }
                    if (w > 0) *at = v;
                    o[d][0] = v.x; o[d][1] = v.y; o[d][2] = v.z; o[d][3] = v.w;
                }
            }
            if (w > 0) consumer_sync();
        }
        if (warp == 0 && alive) {
            if (begins && ends) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = r0 + e * 8, p = t.p0 + r;
                    if (r >= t.rows) continue;
                    const int token = chunk_token(a, p), head = w.head * a.group + p - token * a.group;
                    const long long row = t.row0 + token;
                    const float f = sum[e] == 0.f ? 0.f : 1.f / sum[e];  // (no key: 0)
                    uint16_t* to = a.out + row * a.out_stride + head * HD + c0;
#pragma unroll
                    for (int d = 0; d < HD / 8; ++d) {
                        const uint32_t v = T::pack(o[d][2 * e] * f, o[d][2 * e + 1] * f);
                        if (a.out_vec) {
                            *reinterpret_cast<uint32_t*>(to + d * 8) = v;
                        } else {
                            to[d * 8] = (uint16_t)v;
                            to[d * 8 + 1] = (uint16_t)(v >> 16);
                        }
                    }
                    if (a.lse && (lane & 3) == 0)
                        a.lse[row * (a.kv_heads * a.group) + head] =
                            sum[e] == 0.f ? -INFINITY : LN2 * (mx[e] + log2f(sum[e]));
                }
            } else {
                float* part = a.part + ((size_t)cta * 2 + begins) * TR * (HD + 2);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = r0 + e * 8;
#pragma unroll
                    for (int d = 0; d < HD / 8; ++d)
                        *reinterpret_cast<float2*>(part + r * HD + d * 8 + c0) = make_float2(o[d][2 * e], o[d][2 * e + 1]);
                    if ((lane & 3) == 0)
                        *reinterpret_cast<float2*>(part + TR * HD + 2 * r) = make_float2(mx[e], sum[e]);
                }
            }
        }
    }
}

// ---- merge ----
// Grid (CTA of the kernel before, groups of rows); a warp takes a row of the item that
// begins in that CTA's share and goes on in the next ones': out = sum_c 2^(m_c - M) o_c / L,
// L = sum_c 2^(m_c - M) l_c, M = max m_c, in the CTAs' order, a batch of parts at a time.  Bound by
// latency (the item, then its parts) where items are shared by many CTAs: about 3 us after a
// step; one slot of 32,000 keys and 2 key heads, 125 parts an item, takes 16.6 us a call, 39 with
// the maxima looked for first and four parts at a time.
// Rows of a CTA: most CTAs of the grid have nothing to do, as few items are shared, and for tiles of many rows they are so many
// that they take time (25 prompts, 4, 8, 16, 32 rows: 43.0, 41.6, 41.5, 42.1 us, of 128 dims 70.8, 69.0, 68.2, 69.4); few rows' wait beside the kernel before.
constexpr int merge_rows(int tile_rows) { return tile_rows == FR_ROWS ? 4 : 16; }
template <class T, int HD, int TR>
__global__ void __launch_bounds__(32 * merge_rows(TR)) chunk_merge_kernel(const __grid_constant__ ChunkArgs a) {
    const int cta = blockIdx.x, r = blockIdx.y * merge_rows(TR) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    constexpr int PER = HD / 32, BATCH = TR == FR_ROWS ? 8 : 4;  // (tiles of many rows are shared by few CTAs)
    // (After many rows not: the next call's kernels would start in the merge's way.  Two chunks of thousands of tokens, one call after
    // another: 463 us, 474 with it, 25 prompts 41.5 and 41.8.)
    if (TR == FR_ROWS) pdl_launch_dependents();
    pdl_wait();
    const int* d = a.desc + cta * CH_DESC;
    const int more = d[0];
    if (more <= 0 || r >= d[2]) return;
    constexpr size_t STEP = (size_t)TR * (HD + 2);
    // parts: 1 of `cta` (the item begins there), then 0 of the CTAs after it
    const float* first = a.part + ((size_t)cta * 2 + 1) * STEP;
    const float* rest = a.part + ((size_t)cta + 1) * 2 * STEP;
    auto part = [&](int i) { return i == 0 ? first : rest + (size_t)(i - 1) * 2 * STEP; };
    float top = -INFINITY, sum = 0.f, o[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = 0.f;
    for (int i0 = 0; i0 <= more; i0 += BATCH) {  // a batch's maxima, sums and outputs are on their way together
        float2 x[BATCH], v[BATCH][PER / 2];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const bool there = i0 + i <= more;
            const float* p = part(i0 + i);
            x[i] = there ? *reinterpret_cast<const float2*>(p + TR * HD + 2 * r) : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int e = 0; e < PER / 2; ++e)
                v[i][e] = there ? *reinterpret_cast<const float2*>(p + r * HD + lane * PER + 2 * e) : make_float2(0.f, 0.f);
        }
        float now = top;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) now = fmaxf(now, x[i].x);
        const float ref = now == -INFINITY ? 0.f : now, back = ex2(top - ref);
        top = now;
        sum *= back;
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] *= back;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float f = ex2(x[i].x - ref);
            sum = fmaf(f, x[i].y, sum);
#pragma unroll
            for (int e = 0; e < PER / 2; ++e) {
                o[2 * e] = fmaf(f, v[i][e].x, o[2 * e]);
                o[2 * e + 1] = fmaf(f, v[i][e].y, o[2 * e + 1]);
            }
        }
    }
    const int p = d[1] + r, token = chunk_token(a, p), head = d[4] * a.group + p - token * a.group;
    const long long row = d[3] + token;
    const float f = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t* to = a.out + row * a.out_stride + head * HD + lane * PER;
#pragma unroll
    for (int e = 0; e < PER; e += 2) {
        const uint32_t v = T::pack(o[e] * f, o[e + 1] * f);
        if (a.out_vec) {
            *reinterpret_cast<uint32_t*>(to + e) = v;
        } else {
            to[e] = (uint16_t)v;
            to[e + 1] = (uint16_t)(v >> 16);
        }
    }
    if (a.lse && lane == 0)
        a.lse[row * (a.kv_heads * a.group) + head] = sum == 0.f ? -INFINITY : LN2 * (top + log2f(sum));
}

template <class T, int HD, int TR>
cudaError_t launch_merge(const ChunkArgs& a, cudaStream_t s) {
    return launch_ex(chunk_merge_kernel<T, HD, TR>, dim3(a.ctas, TR / merge_rows(TR)), 32 * merge_rows(TR), 0, s, 1, a);
}
template <class T, int HD>
cudaError_t merge_hd(const ChunkArgs& a, int tile_rows, cudaStream_t s) {
    return tile_rows == FR_ROWS ? launch_merge<T, HD, FR_ROWS>(a, s) : launch_merge<T, HD, 128 * chunk_tc_tiles(HD)>(a, s);
}

// How a call runs: tile rows, CTAs, workspace.
struct ChunkPlan {
    int tile_rows, ctas, max_tiles, min_units;
    bool residues, plan_here;
    size_t start, desc, tiles, part, need;  // places in the workspace, its bytes
};

int chunk_plan(const mtp_chunk_attention_args* a, ChunkPlan* p) {
    if (!a || a->slots < 1 || a->slots > CH_MAX_SLOTS || a->rows < 0 || a->n_heads < 1 || a->n_kv_heads < 1 ||
        a->n_heads % a->n_kv_heads || a->n_heads / a->n_kv_heads > 64 || a->n_heads > 1024)
        return invalid("chunk_attention: invalid sizes (slots, rows or heads)");
    if (a->head_dim != 64 && a->head_dim != 128) return invalid("chunk_attention: head_dim %d: 64 or 128", a->head_dim);
    if (!page_size_ok(a->page_size) || a->layers < 1 || a->layer < 0 || a->layer >= a->layers || a->n_pages < 1 ||
        a->bt_stride < 1 || (long long)a->bt_stride * a->page_size > (1 << 24) ||
        (long long)a->n_pages * a->layers * 2 * a->n_kv_heads > 0x7fffffffLL)
        return invalid("chunk_attention: invalid cache (page_size %d, layers %d, layer %d, pages %d, bt_stride %d)",
                       a->page_size, a->layers, a->layer, a->n_pages, a->bt_stride);
    if (a->dtype != MTP_BF16 && a->dtype != MTP_F16) return invalid("chunk_attention: dtype %d", a->dtype);
    if (a->window < 0 || a->max_new < 0 || a->max_keys < 0 || !(a->scale > 0.f) || !(a->scale < 1e30f))
        return invalid("chunk_attention: window %d, max_new %d, max_keys %d, scale %g", a->window, a->max_new, a->max_keys,
                       (double)a->scale);
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return report_error(MTP_ERR_CUDA, "chunk_attention: no usable CUDA device");
    }
    const int group = a->n_heads / a->n_kv_heads;
    const long long packed = (long long)std::min(a->max_new, a->rows) * group;  // rows of a slot and key head
    p->tile_rows = packed <= FR_ROWS ? FR_ROWS : 128 * chunk_tc_tiles(a->head_dim);
    p->residues = packed <= RESIDUE_ROWS;
    const bool few = p->tile_rows == FR_ROWS;
    const long long tiles = std::min((long long)a->slots * ((packed + p->tile_rows - 1) / p->tile_rows),
                                     (long long)a->rows * group / p->tile_rows + a->slots);
    if ((long long)a->rows * group >= CH_MAX_PACKED)
        return invalid("chunk_attention: %d rows of %d query heads per key head: below %d together", a->rows, group, CH_MAX_PACKED);
    p->max_tiles = (int)tiles;
    const int per_sm = !few ? 3 - chunk_tc_tiles(a->head_dim) : a->head_dim == 64 ? 3 : 2, keys = few ? FR_KEYS : CT_UNIT_KEYS;
    p->min_units = few ? FR_MIN_UNITS : CT_MIN_UNITS;
    const long long units = tiles * a->n_kv_heads * (a->max_keys / keys + 2);
    p->ctas = (int)std::max(1ll, std::min((long long)sms * per_sm, (units + p->min_units - 1) / p->min_units));
    // what a slot can cost at most, in a table of its width, has to fit the plan's 32 bits
    const long long slot_cost = (long long)a->bt_stride * a->page_size / FR_KEYS + 1 + ITEM_COST;
    p->plan_here = few && a->slots <= FR_SLOTS && a->slots * slot_cost * a->n_kv_heads * p->ctas < 1ll << 32;
    auto place = [&](size_t bytes) {
        const size_t at = p->need;
        p->need += (bytes + 255) & ~(size_t)255;
        return at;
    };
    p->need = 0;
    p->start = place((size_t)p->ctas * sizeof(ChunkStart));
    p->desc = place((size_t)p->ctas * CH_DESC * sizeof(int));
    p->tiles = place((size_t)p->max_tiles * sizeof(ChunkTile));
    p->part = place((size_t)p->ctas * 2 * p->tile_rows * (a->head_dim + 2) * sizeof(float));
    return MTP_OK;
}

template <class T, int HD>
cudaError_t launch_rows(const ChunkArgs& a, const CUtensorMap& map, cudaStream_t s) {
    const size_t smem = FrLayout<HD>::BYTES;
    const auto kern = chunk_rows_kernel<T, HD>;
    const cudaError_t e = ensure_kernel_smem(reinterpret_cast<const void*>(kern), smem, true);
    if (e != cudaSuccess) return e;
    return launch_ex(kern, dim3(a.ctas), FR_THREADS, smem, s, 1, a, map);
}
template <class T>
cudaError_t launch_kernels(const ChunkArgs& a, const CUtensorMap& map, const CUtensorMap& q_map, int head_dim, int dtype, int tile_rows, cudaStream_t s) {
    cudaError_t e = a.plan_here ? cudaSuccess : launch_chunk_plan(a, tile_rows, s);
    if (e != cudaSuccess) return e;
    if (tile_rows > FR_ROWS)
        e = launch_chunk_tc(a, map, q_map, head_dim, dtype, s);
    else
        e = head_dim == 64 ? launch_rows<T, 64>(a, map, s) : launch_rows<T, 128>(a, map, s);
    if (e != cudaSuccess) return e;
    return head_dim == 64 ? merge_hd<T, 64>(a, tile_rows, s) : merge_hd<T, 128>(a, tile_rows, s);
}

}  // namespace

}  // namespace mtp

using namespace mtp;

extern "C" {

MTP_API size_t mtp_chunk_attention_workspace_bytes(const mtp_chunk_attention_args* a) {
    size_t need = 0;
    guarded([&]() -> int {
        ChunkPlan p;
        const int r = chunk_plan(a, &p);
        need = r == MTP_OK ? p.need : 0;
        return r;
    });
    return need;
}

MTP_API int mtp_chunk_attention(const mtp_chunk_attention_args* a, void* workspace, size_t workspace_bytes,
                                void* cuda_stream) {
    return guarded([&]() -> int {
        ChunkPlan p;
        if (const int r = chunk_plan(a, &p)) return r;
        const int group = a->n_heads / a->n_kv_heads, width = a->n_heads * a->head_dim;
        if (a->q_stride < width || a->out_stride < width)
            return invalid("chunk_attention: row strides %lld, %lld below %d", (long long)a->q_stride,
                           (long long)a->out_stride, width);
        if (a->rows == 0 || a->max_new == 0) return MTP_OK;  // no new tokens
        if (!a->q || !a->kv_pool || !a->block_table || !a->cu_rows || !a->kv_lens || !a->out)
            return invalid("chunk_attention: null pointer");
        if (!aligned16(a->kv_pool)) return invalid("chunk_attention: kv_pool must be 16-byte aligned");
        if ((reinterpret_cast<uintptr_t>(a->q) | reinterpret_cast<uintptr_t>(a->out)) & 1)
            return invalid("chunk_attention: q and out must be aligned to their elements");
        if (!workspace || !aligned16(workspace) || workspace_bytes < p.need)
            return invalid("chunk_attention: workspace %zu bytes, need %zu, 16-byte aligned", workspace_bytes, p.need);
        ChunkArgs c;
        c.q = static_cast<const uint16_t*>(a->q);
        c.out = static_cast<uint16_t*>(a->out);
        c.lse = a->out_lse;
        c.block_table = a->block_table; c.cu_rows = a->cu_rows; c.kv_lens = a->kv_lens;
        c.q_stride = a->q_stride; c.out_stride = a->out_stride;
        c.slots = a->slots; c.rows = a->rows; c.kv_heads = a->n_kv_heads; c.group = group;
        c.group_inv = group == 1 ? 0u : (uint32_t)(((1ull << 32) + group - 1) / group);
        c.page_shift = a->page_size == 16 ? 4 : a->page_size == 32 ? 5 : a->page_size == 64 ? 6 : 7;
        c.bt_stride = a->bt_stride; c.n_pages = a->n_pages;
        c.page_blocks = a->layers * 2 * a->n_kv_heads;
        c.layer_block = a->layer * 2 * a->n_kv_heads;
        // (no position passes the table: a window as long leaves nothing out, and differences with it stay in 32 bits)
        c.window = a->window < a->bt_stride * a->page_size ? a->window : 0;
        c.max_tiles = p.max_tiles; c.min_units = p.min_units;
        const bool few = p.tile_rows == FR_ROWS;
        c.residues = p.residues;
        c.snap = few ? 0 : CT_SNAP;
        c.plan_here = p.plan_here;
        c.q_vec = aligned16(a->q) && a->q_stride % 8 == 0;
        c.out_vec = aligned16(a->out) && a->out_stride % 8 == 0;
        c.scale_log2 = a->scale * 1.4426950408889634f;
        char* ws = static_cast<char*>(workspace);
        c.ctas = p.ctas;
        c.start = reinterpret_cast<ChunkStart*>(ws + p.start);
        c.desc = reinterpret_cast<int*>(ws + p.desc);
        c.tiles = reinterpret_cast<ChunkTile*>(ws + p.tiles);
        c.part = reinterpret_cast<float*>(ws + p.part);
        c.err = a->err_word;
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        CUtensorMap map, q_map = {};
        if (tc_encode_cache(&map, a->kv_pool, a->dtype, a->head_dim, a->page_size,
                            (uint64_t)a->n_pages * c.page_blocks, std::min(a->page_size, FR_KEYS)) != 0)
            return report_error(MTP_ERR_CUDA, "chunk_attention: cuTensorMapEncodeTiled failed");
        // a tile's 128 packed rows are a box of the query rows where the heads of a key head divide 128
        c.q_tma = !few && c.q_vec && 128 % group == 0 && a->q_stride < (1ll << 38) &&
                  tc_encode_queries(&q_map, a->q, a->dtype, a->head_dim, a->n_heads, a->rows, a->q_stride, group) == 0;
        const cudaError_t e = a->dtype == MTP_BF16 ? launch_kernels<Bf16>(c, map, q_map, a->head_dim, a->dtype, p.tile_rows, s)
                                                   : launch_kernels<F16>(c, map, q_map, a->head_dim, a->dtype, p.tile_rows, s);
        return cuda_status(e, "chunk_attention");
    });
}

}  // extern "C"
