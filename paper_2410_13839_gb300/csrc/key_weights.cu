// key_weights.cu -- the attention weight that each cached key gets from a step's tokens
// (mtp_key_weights): its entry point, the kernel of few rows per slot and key head
// (decoding steps, drafts), and the sum over row segments.
//
//   w_j (+)= sum_p 2^(c q_p . k_j - l_p),  c = scale log2 e, l_p = lse_p log2 e,
//
// over the rows p (tokens and query heads of the key head) that see key j: one product and one
// exponential a pair, no maximum and no second pass, as the log-sum-exps are there.
//
// Few rows: the keys are read once and memory bounds it.  A warp takes 16 keys at a time as M of
// mma.sync (rows as N, eight at a time) straight from global memory into registers: the order of
// the dimensions in a product is free, so a lane's 16 bytes of a key serve two steps of 16, and
// its 16 bytes of a query row, taken in the same order, the same two.  Up to 16 rows (32 of 64 dims) are in registers,
// more in shared memory, as each lane wants them; every warp has several tiles' loads in flight.  A step of 32 slots (180 to 2000 keys, 16 heads of
// 64, 67 MB) takes 15.3 us, 9.9 of which are memory's: a CTA's chain of look-ups (slot, page, keys), about 2.5 us, comes
// before its first byte.  4 drafts on 8 slots of 4,000 to 30,000 keys, 8 key heads of 128 dims (297 MB): 49 to 56 us
// by the GPU, 6.1 to 5.3 TB/s.  8 drafts there (32 rows) 53 to 57, 16 (64 rows) 82: every 16 keys' products read the rows' fragments from
// shared memory again.  One slot alone, 2000 keys of 16 heads of 64 dims, 5.5: 64 CTAs, four rounds of loads in each.
#include <algorithm>

#include "weights.cuh"

namespace mtp {

int tc_encode_cache(CUtensorMap* map, const void* pool, int dtype, int head_dim, int page_size, uint64_t blocks,
                    int box_rows);
int tc_encode_queries(CUtensorMap* map, const void* q, int dtype, int head_dim, int heads, uint64_t rows, uint64_t stride,
                      int group);

namespace {

constexpr int KW_THREADS = 128, KW_WARPS = KW_THREADS / 32;
constexpr int KW_FEW_ROWS = 16, KW_MORE_ROWS = 64;  // packed rows up to which this file's kernel is used; on many keys
template <int HD>
constexpr int KW_HELD_ROWS = HD == 64 ? 32 : 16;  // and up to which their fragments are in registers, else in shared memory

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <class T>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<Bf16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<F16>(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A row tile's part of what the CTA's rows are, in shared memory.
template <int HD>
struct RowTile {
    uint4 q[HD / 32][32];  // each lane's fragments
    float l[8];            // log-sum-exps, times log2 e
    int pos[8];
};
// Grid (chunk of keys and key head, slot).  NT: tiles of eight rows in registers, 0: as many as there are, in shared memory; KT: tiles of 16 keys
// that a warp has in flight.
template <class T, int HD, int NT, int KT>
__global__ void __launch_bounds__(KW_THREADS, NT == 0 ? 5 : 0) key_weights_kernel(const __grid_constant__ WeightsArgs a, int chunk) {
    constexpr int B = HD / 32;  // 16-byte pieces of a row per lane: dimensions 32 b + 8 (lane % 4) .. + 7
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = blockIdx.x / a.kv_heads, head = blockIdx.x - part * a.kv_heads, slot = blockIdx.y;
    pdl_launch_dependents();
    pdl_wait();
    bool cut;
    const WeightsSlot s = weights_slot(a, slot, cut);
    if (cut && a.err && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.err, ERR_BOUNDS);
    const int rows = s.n * a.group, first = part * chunk, last = min(min(s.len, a.keys), first + chunk);
    if (rows == 0 || first >= last) return;
    const int lowest = a.window > 0 ? max(0, s.base - a.window + 1) : 0;  // the first key that some row sees
    if (last <= lowest) return;

    // the rows: fragments, log-sum-exps and positions of columns 2 (lane % 4), + 1 of every tile
    const int tiles = NT > 0 ? NT : (rows + 7) >> 3;
    auto fragment = [&](int t, int b) {
        const int p = t * 8 + (lane >> 2), token = p / a.group;
        const uint16_t* src = a.q + (long long)(s.row0 + token) * a.q_stride + (head * a.group + p - token * a.group) * HD + (lane & 3) * 8;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (p < rows) {
            if (a.q_vec) {
                v = *reinterpret_cast<const uint4*>(src + b * 32);
            } else {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = (uint32_t)src[b * 32 + 2 * e] | (uint32_t)src[b * 32 + 2 * e + 1] << 16;
                v = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        return v;
    };
    auto column = [&](int c, float& l, int& pos) {
        const int token = c / a.group;
        l = 0.f;
        pos = -1;
        if (c < rows) {
            l = a.lse[(long long)(s.row0 + token) * (a.kv_heads * a.group) + head * a.group + c - token * a.group] * LOG2E;
            pos = s.base + token;
        }
    };
    constexpr int HELD = NT > 0 ? NT : 1;
    uint4 q[HELD][B];
    float l[HELD][2];
    int pos[HELD][2];
    extern __shared__ __align__(16) unsigned char kw_sm[];
    RowTile<HD>* row_tiles = reinterpret_cast<RowTile<HD>*>(kw_sm);
    if constexpr (NT > 0) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int b = 0; b < B; ++b) q[t][b] = fragment(t, b);
#pragma unroll
            for (int e = 0; e < 2; ++e) column(t * 8 + (lane & 3) * 2 + e, l[t][e], pos[t][e]);
        }
    } else {
        for (int t = warp; t < tiles; t += KW_WARPS) {
#pragma unroll
            for (int b = 0; b < B; ++b) row_tiles[t].q[b][lane] = fragment(t, b);
            if (lane < 8) column(t * 8 + lane, row_tiles[t].l[lane], row_tiles[t].pos[lane]);
        }
        __syncthreads();
    }
    const int* table = a.block_table + (size_t)slot * a.bt_stride;
    float* out = a.weights + slot * a.w_slot + (long long)head * a.width;
    const int r = lane >> 2, end = s.base + s.n;  // this lane's keys r, r + 8 of a tile
    const int from = max(first, lowest & ~15);
    for (int key0 = from + warp * 16 * KT; key0 < last; key0 += KW_WARPS * 16 * KT) {
        uint4 k[KT][2][B];
        float old[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            const int key = key0 + j * 16;
            const int page = key < last ? table[key >> a.page_shift] : -1;
            const bool there = page >= 0 && page < a.n_pages;
            const uint16_t* src = a.pool + ((((long long)page * a.page_blocks + a.layer_block + head) << a.page_shift) + (key & ((1 << a.page_shift) - 1)) + r) * HD + (lane & 3) * 8;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int b = 0; b < B; ++b)
                    k[j][h][b] = there ? *reinterpret_cast<const uint4*>(src + h * 8 * HD + b * 32) : make_uint4(0u, 0u, 0u, 0u);
            const int mine = key + r + (lane & 1) * 8;
            old[j] = (lane & 3) < 2 && mine < last && mine < s.base ? out[mine] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            const int key = key0 + j * 16;
            if (key >= last) break;
            float sum[2] = {0.f, 0.f};
            const bool seen = key + 15 <= s.base && (a.window <= 0 || key > end - 1 - a.window);  // by every row
            auto add = [&](const uint4 (&rows_q)[B], const float (&rows_l)[2], const int (&rows_pos)[2], bool inner) {
                float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    const uint4 x = k[j][0][b], y = k[j][1][b], z = rows_q[b];
                    mma16<T>(d, x.x, y.x, x.y, y.y, z.x, z.y);
                    mma16<T>(d, x.z, y.z, x.w, y.w, z.z, z.w);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float w = ex2(fmaf(d[2 * h + e], a.scale_log2, -rows_l[e]));
                        const int at = key + r + h * 8;
                        if (!inner && (at > rows_pos[e] || (a.window > 0 && at <= rows_pos[e] - a.window))) w = 0.f;
                        sum[h] += w;
                    }
            };
            if constexpr (NT > 0) {
                const bool inner = seen && rows == NT * 8;
#pragma unroll
                for (int t = 0; t < NT; ++t) add(q[t], l[t], pos[t], inner);
            } else {
#pragma unroll 2
                for (int t = 0; t < tiles; ++t) {
                    const RowTile<HD>& x = row_tiles[t];
#pragma unroll
                    for (int b = 0; b < B; ++b) q[0][b] = x.q[b][lane];
                    const float2 y = *reinterpret_cast<const float2*>(x.l + (lane & 3) * 2);
                    const int2 z = *reinterpret_cast<const int2*>(x.pos + (lane & 3) * 2);
                    l[0][0] = y.x; l[0][1] = y.y;
                    pos[0][0] = z.x; pos[0][1] = z.y;
                    add(q[0], l[0], pos[0], seen && t * 8 + 8 <= rows);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                sum[h] += __shfl_xor_sync(FULL_MASK, sum[h], 1);
                sum[h] += __shfl_xor_sync(FULL_MASK, sum[h], 2);
            }
            const int mine = key + r + (lane & 1) * 8;
            if ((lane & 3) < 2 && mine < last && mine >= lowest) out[mine] = old[j] + (lane & 1 ? sum[1] : sum[0]);
        }
    }
}

// The segments' sums, in their order, onto what the keys had.  Grid (keys / 256, key head, slot).
__global__ void __launch_bounds__(256) key_weights_sum_kernel(const __grid_constant__ WeightsArgs a) {
    const int key = blockIdx.x * 256 + threadIdx.x, head = blockIdx.y, slot = blockIdx.z;
    pdl_launch_dependents();
    pdl_wait();
    bool cut;
    const WeightsSlot s = weights_slot(a, slot, cut);
    const int lowest = a.window > 0 ? max(0, s.base - a.window + 1) : 0;
    if (s.n == 0 || key >= min(s.len, a.keys) || key < lowest) return;
    float* out = a.weights + slot * a.w_slot + (long long)head * a.width + key;
    float w = key < s.base ? *out : 0.f;
    const size_t step = (size_t)a.slots * a.kv_heads * a.width;
    const float* part = a.part + ((size_t)slot * a.kv_heads + head) * a.width + key;
    float sum = 0.f;
    for (int i = 0; i < a.segments; ++i) sum += part[i * step];
    *out = w + sum;
}

// How a call runs.
struct WeightsPlan {
    bool few;
    int group, key_tiles, tiles, segments;
    size_t need;
};
constexpr int KW_TILE = 128;

int weights_plan(const mtp_key_weights_args* a, WeightsPlan* p) {
    if (!a || a->slots < 1 || a->slots > KW_MAX_SLOTS || a->rows < 0 || a->n_heads < 1 || a->n_kv_heads < 1 ||
        a->n_heads % a->n_kv_heads || a->n_heads / a->n_kv_heads > 64 || a->n_heads > 1024)
        return invalid("key_weights: invalid sizes (slots, rows or heads)");
    if (a->head_dim != 64 && a->head_dim != 128) return invalid("key_weights: head_dim %d: 64 or 128", a->head_dim);
    if (!page_size_ok(a->page_size) || a->layers < 1 || a->layer < 0 || a->layer >= a->layers || a->n_pages < 1 ||
        a->bt_stride < 1 || (long long)a->bt_stride * a->page_size > (1 << 24) ||
        (long long)a->n_pages * a->layers * 2 * a->n_kv_heads > 0x7fffffffLL)
        return invalid("key_weights: invalid cache (page_size %d, layers %d, layer %d, pages %d, bt_stride %d)",
                       a->page_size, a->layers, a->layer, a->n_pages, a->bt_stride);
    if (a->dtype != MTP_BF16 && a->dtype != MTP_F16) return invalid("key_weights: dtype %d", a->dtype);
    if (a->window < 0 || a->max_new < 0 || a->max_keys < 0 || !(a->scale > 0.f) || !(a->scale < 1e30f))
        return invalid("key_weights: window %d, max_new %d, max_keys %d, scale %g", a->window, a->max_new, a->max_keys,
                       (double)a->scale);
    p->group = a->n_heads / a->n_kv_heads;
    if ((long long)a->rows * p->group >= 1 << 21)
        return invalid("key_weights: %d rows of %d query heads per key head: below %d together", a->rows, p->group, 1 << 21);
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return report_error(MTP_ERR_CUDA, "key_weights: no usable CUDA device");
    }
    const long long width = (long long)a->bt_stride * a->page_size;
    const long long packed = (long long)std::min(a->max_new, a->rows) * p->group;  // rows of a slot and key head
    p->key_tiles = (int)((std::min((long long)a->max_keys, width) + KW_TILE - 1) / KW_TILE);
    const long long lists = (long long)a->slots * a->n_kv_heads, row_tiles = (packed + KW_TILE - 1) / KW_TILE;
    const bool much = lists * p->key_tiles >= 8 * sms;  // work for all SMs
    // This file's kernel and tcgen05, us: 24, 36, 64 rows of 128 dims on 8 contexts of 4,000 to 30,000 keys, 8 key heads, 53, 125; 65, 130; 83, 136;
    // 32, 36, 64 rows on 32 of up to 2000 23, 40; 26, 43; 35, 44; 64 rows on 4 of up to 8000 34, 27.  Too few keys for all SMs: 32 rows on one
    // context of 2000, 4 key heads, 12.4, 5.1
    p->few = packed <= KW_FEW_ROWS || (packed <= KW_MORE_ROWS && much && p->key_tiles >= 8);
    p->segments = p->tiles = 1;
    p->need = 0;
    if (!p->few) {
        // four key tiles of a CTA read the rows from L2 a quarter as often: for long contexts that have work for all SMs.  One, four: two
        // chunks after 6000 to 9000 keys 607, 484 us, 8 slots of 9 new tokens and up to 16000 keys 57, 44; 25 prompts of up to
        // 578 tokens 41.5, 51.8, one chunk of 2000 tokens after 4000, one key head, 37.7, 42.9
        p->tiles = p->key_tiles >= 16 && much ? 4 : 1;
        // few keys and many rows: the rows are cut too, until every SM has work enough
        const long long groups = std::max(1ll, lists * ((p->key_tiles + p->tiles - 1) / p->tiles));
        p->segments = (int)std::max(1ll, std::min((row_tiles + 3) / 4, (8ll / (p->tiles == 4 ? 1 : 2) * sms + groups / 2) / groups));
        if (p->segments > 1) p->need = (size_t)p->segments * a->slots * a->n_kv_heads * width * sizeof(float);
    }
    return MTP_OK;
}

template <class T, int HD>
cudaError_t launch_few(const WeightsArgs& a, cudaStream_t s) {
    const int packed = std::min(a.max_new, a.rows) * a.group;
    // Tiles in flight, and how often: once, twice, four and eight times two tiles 18.9, 15.9, 15.4, 18.7 us (a step of 32 slots) and 63, 52, 49, 50
    // (4 drafts on 8 long contexts); four tiles of 64 dims 17 to 22, of 128 dims 74, one of 128 dims 52 at best.
    constexpr int chunk = KW_WARPS * 16 * 8;
    const dim3 grid((a.keys + chunk - 1) / chunk * a.kv_heads, a.slots);
    // Rows in shared memory: 17 to 32 of 128 dims on 8 contexts of 4,000 to 30,000 keys 53 us, in registers (two or four CTAs an SM) 96, 73; of
    // 64 dims on 32 of up to 2000 13.0 and 11.3, on the long ones 25.5 and 27.1.
    const bool held = packed <= KW_HELD_ROWS<HD>;
    auto kern = packed <= 8 ? key_weights_kernel<T, HD, 1, 2> : packed <= 16 ? key_weights_kernel<T, HD, 2, 2> : key_weights_kernel<T, HD, 0, 1>;
    if constexpr (HD == 64)
        if (packed > 16 && held) kern = key_weights_kernel<T, HD, 4, 2>;
    return launch_ex(kern, grid, KW_THREADS, held ? 0 : (size_t)(packed + 7) / 8 * sizeof(RowTile<HD>), s, 1, a, chunk);
}

}  // namespace
}  // namespace mtp

using namespace mtp;

extern "C" {

MTP_API size_t mtp_key_weights_workspace_bytes(const mtp_key_weights_args* a) {
    size_t need = 0;
    guarded([&]() -> int {
        WeightsPlan p;
        const int r = weights_plan(a, &p);
        need = r == MTP_OK ? p.need : 0;
        return r;
    });
    return need;
}

MTP_API int mtp_key_weights(const mtp_key_weights_args* a, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return guarded([&]() -> int {
        WeightsPlan p;
        if (const int r = weights_plan(a, &p)) return r;
        if (a->q_stride < a->n_heads * a->head_dim)
            return invalid("key_weights: row stride %lld below %d", (long long)a->q_stride, a->n_heads * a->head_dim);
        if (a->rows == 0 || a->max_new == 0 || a->max_keys == 0) return MTP_OK;  // no new tokens
        if (!a->q || !a->kv_pool || !a->block_table || !a->cu_rows || !a->kv_lens || !a->lse || !a->weights)
            return invalid("key_weights: null pointer");
        if (!aligned16(a->kv_pool)) return invalid("key_weights: kv_pool must be 16-byte aligned");
        if (reinterpret_cast<uintptr_t>(a->q) & 1 || (reinterpret_cast<uintptr_t>(a->lse) | reinterpret_cast<uintptr_t>(a->weights)) & 3)
            return invalid("key_weights: q, lse and weights must be aligned to their elements");
        if (p.need > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < p.need))
            return invalid("key_weights: workspace %zu bytes, need %zu, 16-byte aligned", workspace_bytes, p.need);
        WeightsArgs w;
        w.q = static_cast<const uint16_t*>(a->q);
        w.pool = static_cast<const uint16_t*>(a->kv_pool);
        w.block_table = a->block_table; w.cu_rows = a->cu_rows; w.kv_lens = a->kv_lens; w.lse = a->lse;
        w.width = a->bt_stride * a->page_size;
        w.weights = a->weights + (size_t)a->layer * a->n_kv_heads * w.width;
        w.w_slot = (long long)a->layers * a->n_kv_heads * w.width;
        w.q_stride = a->q_stride;
        w.slots = a->slots; w.rows = a->rows; w.kv_heads = a->n_kv_heads; w.group = p.group; w.dim = a->head_dim;
        w.page_shift = log2_of(a->page_size);
        w.bt_stride = a->bt_stride; w.n_pages = a->n_pages;
        w.page_blocks = a->layers * 2 * a->n_kv_heads;
        w.layer_block = a->layer * 2 * a->n_kv_heads;
        // (no position passes the table: a window as long leaves nothing out, and sums with it stay in 32 bits)
        w.window = a->window < w.width ? a->window : 0;
        w.max_new = a->max_new;
        w.keys = std::min(a->max_keys, w.width);
        w.tiles = p.tiles;
        w.segments = p.segments;
        w.part = static_cast<float*>(workspace);
        w.q_vec = aligned16(a->q) && a->q_stride % 8 == 0;
        w.scale_log2 = a->scale * LOG2E;
        w.err = a->err_word;
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        if (p.few) {
            auto few = [&](auto type) {
                using T = decltype(type);
                return a->head_dim == 64 ? launch_few<T, 64>(w, s) : launch_few<T, 128>(w, s);
            };
            return cuda_status(a->dtype == MTP_BF16 ? few(Bf16{}) : few(F16{}), "key_weights");
        }
        CUtensorMap map, q_map = {};
        if (tc_encode_cache(&map, a->kv_pool, a->dtype, a->head_dim, a->page_size, (uint64_t)a->n_pages * w.page_blocks,
                            std::min(a->page_size, KW_TILE)) != 0)
            return report_error(MTP_ERR_CUDA, "key_weights: cuTensorMapEncodeTiled failed");
        const bool q_tma = w.q_vec && a->q_stride < (1ll << 38) &&
                           tc_encode_queries(&q_map, a->q, a->dtype, a->head_dim, a->n_heads, a->rows, a->q_stride, p.group) == 0;
        cudaError_t e = launch_weights_tc(w, map, q_map, q_tma, a->dtype, p.key_tiles, s);
        if (e == cudaSuccess && p.segments > 1)
            e = launch_ex(key_weights_sum_kernel, dim3((w.keys + 255) / 256, w.kv_heads, w.slots), 256, 0, s, 1, w);
        return cuda_status(e, "key_weights");
    });
}

}  // extern "C"
