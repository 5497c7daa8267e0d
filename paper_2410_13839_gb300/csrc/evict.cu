// evict.cu -- contexts brought down to a budget of keys (mtp_cache_evict): of every slot, layer and
// key head the keys of largest weight stay, beside the first and the last ones, move up in their
// order, and the pages behind them become free.
//
// A CTA has one (slot, layer, key head).  It selects: the weights are in shared memory, as
// whole numbers in the order of the weights, and the m-th largest is found by its highest 11 bits, the 11
// after them and the last 10, each time by counting how many keys have each value; few keys that share the
// first bits are compared with each other instead.  Of the keys
// equal to it the first ones stay.  Ballots and prefix sums then give each key that stays its place, and a list
// of their rows in the pool takes the weights' place.
// Then it moves keys and values in place: it goes through its list from the front, a stage of rows at a
// time: read, barrier, write.  Row j is read from place old_j >= j, and places before a stage's are never read
// again, so that no copy of the cache is needed; further stages are on their way into shared memory
// meanwhile.  Memory bounds it: one CTA's selection lies behind another's moves.  A small kernel before looks at
// the tables: no count changes before every page has been looked at.
// 16 slots of 180 to 2000 keys cut to 700, 12 layers of 16 heads of 64 (773 MB): 136 us (133 to 150 by the GPU), 5.7 TB/s; four contexts of
// 20,000 to 30,000 cut to 8192, 4 layers of 8 heads of 128 (1.08 GB): 190 us, of which the selection, which all 128 CTAs
// make at the same time, about 25; one utterance, 1088 keys cut to 1024 (102 MB): 27 us, 8 of them before the first row moves.
// (Found bit by bit, with 32 counts, the selections took 16, 126 and 67 us of their own; from registers, 16 to 64
// keys a thread, the unrolled code did not stay in the instruction cache.)
#include <algorithm>
#include <climits>

#include "serving.cuh"

namespace mtp {
namespace {

constexpr int EV_BINS = 2048;
constexpr int EV_HELD = 32768;   // keys whose order shared memory holds
constexpr int EV_SMEM = 231424;  // shared memory of a CTA that has an SM to itself
constexpr int EV_FEW = 256;      // keys of a border's bin that are compared with each other
constexpr int EV_STAGES = 4;     // of rows on their way into shared memory: 3, 4, 6 take 140, 139, 147 us for 16 slots of 12 layers

struct EvictArgs {
    mtp_cache_evict_args a;
    int shift;      // page_size = 1 << shift
    int width;      // bt_stride * page_size: weights of a slot, layer and head
    int heads;      // layers * n_kv_heads
    int smem;       // bytes of shared memory
    bool vector;    // weights on 16-byte boundaries
    int* list;      // workspace [slots][layers][heads][width], of wide tables: row of the pool (page * page_size + offset) of each key that stays
};

// A slot: keys before and after, the first and last ones that stay whatever their weight.
struct EvictSlot {
    int len, after, sinks, recent;
};
__device__ __forceinline__ EvictSlot evict_slot(const mtp_cache_evict_args& a, int slot) {
    EvictSlot s;
    s.len = a.kv_lens[slot];
    s.after = min(s.len, a.keep[slot]);
    s.sinks = min(s.after, a.sinks);
    s.recent = min(s.after - s.sinks, a.recent);
    return s;
}

// Weights as whole numbers above 0 in their order; NaN above all, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float w) {
    const uint32_t b = w == 0.f ? 0u : __float_as_uint(w);
    return w != w ? 0xffffffffu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// What can be said of a slot without its weights: whether it may be changed, its table and length afterwards.  Copies the
// counts, where they go to another array.
constexpr int EC_THREADS = 1024;
__global__ void __launch_bounds__(EC_THREADS) evict_check_kernel(const __grid_constant__ EvictArgs p) {
    const mtp_cache_evict_args& a = p.a;
    const int tid = threadIdx.x, slot = blockIdx.x, mask = (1 << p.shift) - 1;
    pdl_launch_dependents();
    pdl_wait();
    if (a.out_page_refs != a.page_refs)
        for (int i = slot * EC_THREADS + tid; i < a.n_pages; i += gridDim.x * EC_THREADS) a.out_page_refs[i] = a.page_refs[i];
    if (slot >= a.slots) return;
    const EvictSlot s = evict_slot(a, slot);
    const int* table = a.block_table + (long long)slot * a.bt_stride;
    bool bad = s.len < 0 || s.len > p.width || a.keep[slot] < 0;
    const int written = (s.after + mask) >> p.shift;
    if (!bad && s.after < s.len) {
        // every held page is one and is counted; those that are written, if a key stays behind the sinks, are in no other table
        const int held = (s.len + mask) >> p.shift, same = s.after > s.sinks ? s.sinks >> p.shift : written;
#pragma unroll 4
        for (int c = tid; c < held; c += EC_THREADS) {
            const int page = table[c], n = page >= 0 && page < a.n_pages ? a.page_refs[page] : 0;
            bad |= n < 1 || (n > 1 && c >= same && c < written);
        }
    }
    bad = __syncthreads_or(bad) != 0;
    const int used = bad ? a.bt_stride : written;
    for (int c = tid; c < a.bt_stride; c += EC_THREADS) a.out_block_table[(long long)slot * a.bt_stride + c] = c < used ? table[c] : -1;
    if (tid == 0) {
        a.out_kv_lens[slot] = bad ? s.len : s.after;
        a.out_status[slot] = bad ? MTP_ERR_INVALID : MTP_OK;
    }
}

__device__ __forceinline__ void copy16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(dst)), "l"(src) : "memory");
}
// The rows of a list (row of the pool of each key that stays, in their order) to their places, of one layer and head: keys, values or both.  A
// thread has a fixed 16-byte piece of a row, in every UNROLL * (threads / pieces)-th row; it writes what it has read itself, so
// that the stages need no barrier of their own.
template <int NT, int UNROLL>
__device__ __forceinline__ void move_rows(const EvictArgs& p, const EvictSlot& s, const int* table, const int* list, uint4* ring, int layer, int head,
                                          int kv0, int kvs) {
    const mtp_cache_evict_args& a = p.a;
    const int tid = threadIdx.x, mask = (1 << p.shift) - 1;
    const int vecs = a.head_dim / 8, pieces = vecs * kvs, rows = NT / pieces, r0 = tid / pieces, v = tid - r0 * pieces, step = rows * UNROLL;
    const bool active = r0 < rows;
    // a piece of row `row` (page * page_size + offset): the pool's blocks of a page apart, the head's among them
    const int kv = kv0 + v / vecs;
    uint4* pool = static_cast<uint4*>(a.kv_pool) + ((((long long)layer * 2 + kv) * a.n_kv_heads + head) << p.shift) * vecs + v % vecs;
    const long long page_step = ((long long)p.heads * 2 << p.shift) * vecs;
    auto at = [&](int page, int offset) { return pool + page * page_step + offset * vecs; };
    int from[UNROLL];  // rows of the stage that is asked for next, on their way
    auto look = [&](int j0) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int j = j0 + u * rows + r0;
            from[u] = active && j < s.after ? list[j] : -1;
        }
    };
    auto ask = [&](int stage) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
            if (from[u] >= 0) copy16(ring + (stage * UNROLL + u) * NT + tid, at(from[u] >> p.shift, from[u] & mask));
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int next = s.sinks;  // (the first rows stay where they are)
    look(next);
#pragma unroll 1
    for (int k = 0; k < EV_STAGES - 1; ++k) {
        ask(k);
        look(next += step);
    }
    int in = EV_STAGES - 1, out = 0;
#pragma unroll 1
    for (int j0 = s.sinks; j0 < s.after; j0 += step) {
        int to[UNROLL];  // (looked up before the stores, which might change the table for all that the compiler knows)
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int j = j0 + u * rows + r0;
            to[u] = active && j < s.after ? table[j >> p.shift] : -1;
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(EV_STAGES - 2) : "memory");
        __syncthreads();  // every row of this stage and the ones before is read
        ask(in);
        look(next += step);
        uint4 piece[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) piece[u] = ring[(out * UNROLL + u) * NT + tid];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
            if (to[u] >= 0) *at(to[u], (j0 + u * rows + r0) & mask) = piece[u];
        in = in + 1 == EV_STAGES ? 0 : in + 1;
        out = out + 1 == EV_STAGES ? 0 : out + 1;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}
// the slot's pages that become free
template <int NT>
__device__ __forceinline__ void free_pages(const EvictArgs& p, const EvictSlot& s, const int* table) {
    const int mask = (1 << p.shift) - 1;
    for (int c = ((s.after + mask) >> p.shift) + threadIdx.x; c < (s.len + mask) >> p.shift; c += NT) atomicSub(p.a.out_page_refs + table[c], 1);
}

constexpr size_t ring_bytes(int threads, int unroll) { return (size_t)EV_STAGES * unroll * threads * 16; }

// Selection, and the moves: grid (run, its parts).  HELD: the weights' order is kept in shared memory, where the list takes its place, and the
// CTA moves the rows (of keys and values, or one part's); else (rows past EV_HELD keys) the order is made again in every pass, and the list
// goes to the workspace.
template <int NT, bool HELD, int UNROLL, int CTAS>
__global__ void __launch_bounds__(NT, CTAS) evict_kernel(const __grid_constant__ EvictArgs p) {
    constexpr int WARPS = NT / 32, B = EV_BINS / NT, BATCH = NT == 1024 ? 8 : 4;
    extern __shared__ __align__(16) unsigned char ev_sm[];  // the order of the weights, then the list; behind them the counts of a pass, then the ring
    __shared__ uint32_t part[WARPS], tied_of[2][WARPS], kept_of[2][WARPS];
    __shared__ int s_bin, s_left, s_count, s_few;
    __shared__ uint32_t s_border;
    uint32_t* keys = reinterpret_cast<uint32_t*>(ev_sm);
    uint32_t* bins = keys + (HELD ? p.width : 0);  // (widths are multiples of 16)
    const mtp_cache_evict_args& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int run = blockIdx.x, sub = blockIdx.y, slot = run / p.heads, rest = run - slot * p.heads;
    pdl_launch_dependents();
    for (int i = tid; i < EV_BINS; i += NT) bins[i] = 0;
    if (tid == 0) s_few = 0;
    pdl_wait();
    const EvictSlot s = evict_slot(a, slot);
    const bool moves = a.out_status[slot] == MTP_OK && s.after < s.len;
    const float* w = a.weights + (long long)run * p.width;
    float* out = a.out_weights + (long long)run * p.width;
    if (!moves) {
        if (sub == 0)
            for (int i = tid; i < min(max(s.len, 0), p.width); i += NT) out[i] = w[i];
        return;
    }
    const int mask = (1 << p.shift) - 1;
    const int* table = a.block_table + (long long)slot * a.bt_stride;
    if (HELD && rest == 0 && sub == 0) free_pages<NT>(p, s, table);
    const int lo = s.sinks, hi = s.len - s.recent, want = s.after - s.sinks - s.recent;  // of keys [lo, hi) so many
    auto order_at = [&](int at) { return at >= lo && at < hi ? order_of(w[at]) : 0u; };  // 0: not to be chosen
    if (HELD && p.vector) {
#pragma unroll 4
        for (int i = tid * 4; i < s.len; i += NT * 4) {  // (rows are multiples of 16 long)
            const float4 x = *reinterpret_cast<const float4*>(w + i);
            auto order = [&](int at, float y) { return at >= lo && at < hi ? order_of(y) : 0u; };
            *reinterpret_cast<uint4*>(keys + i) = make_uint4(order(i, x.x), order(i + 1, x.y), order(i + 2, x.z), order(i + 3, x.w));
        }
    } else if (HELD) {
#pragma unroll 4
        for (int i = tid; i < s.len; i += NT) keys[i] = order_at(i);
    }
    __syncthreads();
    auto key_at = [&](int at) { return at >= s.len ? 0u : HELD ? keys[at] : order_at(at); };

    // the want-th largest, from its highest bits: how many keys have each value of the next 11 bits
    uint32_t border = 0;
    int left = want;   // keys that stay of those on the border
    bool all = false;  // all of those on the border stay
    if (want > 0)
#pragma unroll 1
        for (int shift = 21, width = 11; !all;) {
#pragma unroll 1
            for (int i0 = tid; i0 < s.len; i0 += NT * 4) {
                uint32_t key[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) key[e] = key_at(i0 + e * NT);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (key[e] != 0 && (shift == 21 || (key[e] ^ border) >> (shift + width) == 0))
                        atomicAdd(&bins[key[e] >> shift & ((1u << width) - 1)], 1u);
            }
            __syncthreads();
            // the bin that the left-th largest is in: sums from the highest bin down, B bins a thread
            uint32_t mine[B], sum = 0;
            const int bin0 = EV_BINS - B * (tid + 1);
#pragma unroll
            for (int i = 0; i < B; i += 2) {
                uint2* two = reinterpret_cast<uint2*>(bins + bin0 + i);
                const uint2 x = *two;
                *two = make_uint2(0u, 0u);
                mine[i] = x.x;
                mine[i + 1] = x.y;
                sum += x.x + x.y;
            }
            uint32_t x = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(FULL_MASK, x, o);
                if (lane >= o) x += u;
            }
            if (lane == 31) part[warp] = x;
            __syncthreads();
            uint32_t before = __reduce_add_sync(FULL_MASK, lane < warp ? part[lane] : 0u) + x - sum;
            if (before < (uint32_t)left && before + sum >= (uint32_t)left) {
#pragma unroll
                for (int i = B - 1; i >= 0; --i) {
                    if (before < (uint32_t)left && before + mine[i] >= (uint32_t)left) {
                        s_bin = bin0 + i;
                        s_left = left - (int)before;
                        s_count = (int)mine[i];
                    }
                    before += mine[i];
                }
            }
            __syncthreads();
            border |= (uint32_t)s_bin << shift;
            left = s_left;
            all = s_count == left;
            if (shift == 0) break;
            // Few: one utterance 29.8 -> 26.6 us, four long contexts 194.6 -> 190.3.  With 256 threads the code around it gets slower, the 16
            // slots 136 -> 147.
            if (const int n = s_count; NT > 256 && !all && n <= EV_FEW) {  // each one's place among them (the counts are 0 again)
#pragma unroll 1
                for (int i0 = warp * 32; i0 < s.len; i0 += NT) {
                    const uint32_t key = key_at(i0 + lane);
                    if (key != 0 && (key ^ border) >> shift == 0) bins[atomicAdd(&s_few, 1)] = key;
                }
                __syncthreads();
                if (tid < n) {
                    const uint32_t key = bins[tid];
                    int above = 0, alike = 0;
#pragma unroll 2
                    for (int j = 0; j < n; j += 4) {
                        const uint4 x = *reinterpret_cast<const uint4*>(bins + j);
                        above += (x.x > key) + (x.y > key) + (x.z > key) + (x.w > key);
                        alike += (x.x == key) + (x.y == key) + (x.z == key) + (x.w == key);
                    }
                    if (above < left && above + alike >= left) {
                        s_border = key;
                        s_left = left - above;
                        s_count = alike;
                    }
                }
                __syncthreads();
                border = s_border;
                left = s_left;
                all = s_count == left;
                break;
            }
            width = shift == 21 ? 11 : 10;
            shift -= width;
        }
    // Keys NT * BATCH at a time, in their order, a warp's in one piece: how many of each warp stay, then their places.  A key goes to a
    // place at or before its own, and the ones of a segment are read before any is written.
    const bool ties = want > 0 && !all;  // of the keys on the border only the first `left` stay
    border = want > 0 ? max(border, 1u) : 0xffffffffu;
    auto sure = [&](int at, uint32_t key) {
        return at < lo || (at >= hi && at < s.len) || (want > 0 && (ties ? key > border : key >= border));
    };
    int* list = HELD ? reinterpret_cast<int*>(keys) : p.list + (long long)run * p.width;
    const unsigned below = (1u << lane) - 1;
    int place = 0;
    for (int i0 = 0, turn = 0; i0 < s.len; i0 += NT * BATCH, turn ^= 1) {
        const int mine = i0 + warp * 32 * BATCH + lane;
        uint32_t key[BATCH];
        int n_sure = 0, n_tied = 0;
        const bool any = i0 + warp * 32 * BATCH < s.len;  // (of the warp)
        if (any)
#pragma unroll
            for (int e = 0; e < BATCH; ++e) {
                key[e] = key_at(mine + e * 32);
                n_sure += __popc(__ballot_sync(FULL_MASK, sure(mine + e * 32, key[e])));
                if (ties) n_tied += __popc(__ballot_sync(FULL_MASK, key[e] == border));
            }
        if (lane == 0) {
            kept_of[turn][warp] = n_sure;
            tied_of[turn][warp] = n_tied;
        }
        __syncthreads();
        const int sure_all = lane < WARPS ? (int)kept_of[turn][lane] : 0, tied_all = lane < WARPS ? (int)tied_of[turn][lane] : 0;
        const int tied_before = __reduce_add_sync(FULL_MASK, lane < warp ? tied_all : 0), tied = __reduce_add_sync(FULL_MASK, tied_all);
        int to = place + __reduce_add_sync(FULL_MASK, lane < warp ? sure_all : 0) + (ties ? min(tied_before, left) : 0);
        int take = max(0, left - tied_before);
        place += __reduce_add_sync(FULL_MASK, sure_all) + (ties ? min(tied, left) : 0);
        left = max(0, left - tied);
        if (!any) continue;
        int dst[BATCH], page[BATCH];
        float weight[BATCH];
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            const int at = mine + e * 32;
            bool keep = sure(at, key[e]);
            if (ties) {
                const unsigned tied = __ballot_sync(FULL_MASK, key[e] == border);
                keep |= key[e] == border && __popc(tied & below) < take;
                take = max(0, take - __popc(tied));
            }
            const unsigned kept = __ballot_sync(FULL_MASK, keep);
            dst[e] = keep ? to + __popc(kept & below) : -1;
            to += __popc(kept);
            page[e] = keep ? table[at >> p.shift] : 0;
            // the weight is in its order but for the sign of 0 and NaN's bits, and where there is none
            const bool plain = key[e] != 0 && key[e] != 0x80000000u && key[e] != 0xffffffffu;
            weight[e] = plain ? __uint_as_float(key[e] & 0x80000000u ? key[e] ^ 0x80000000u : ~key[e]) : keep ? w[at] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            if (dst[e] < 0) continue;
            if (sub == 0) out[dst[e]] = weight[e];
            list[dst[e]] = (page[e] << p.shift) + ((mine + e * 32) & mask);
        }
    }
    if (!HELD) return;
    __syncthreads();  // the list is there
    const int layer = rest / a.n_kv_heads, head = rest - layer * a.n_kv_heads;
    // the ring has what the list leaves: twice the rows a stage where that is enough
    const int begin = (s.after * 4 + 15) & ~15, kvs = gridDim.y == 1 ? 2 : 1;
    uint4* ring = reinterpret_cast<uint4*>(ev_sm + begin);
    if (begin + (int)ring_bytes(NT, 2 * UNROLL) <= p.smem)
        move_rows<NT, 2 * UNROLL>(p, s, table, list, ring, layer, head, sub, kvs);
    else
        move_rows<NT, UNROLL>(p, s, table, list, ring, layer, head, sub, kvs);
}

// The moves of a list in the workspace.  Grid (run * 2 + keys | values).
constexpr int EM_THREADS = 256, EM_UNROLL = 4;
__global__ void __launch_bounds__(EM_THREADS) evict_move_kernel(const __grid_constant__ EvictArgs p) {
    extern __shared__ __align__(16) unsigned char ev_sm[];
    const mtp_cache_evict_args& a = p.a;
    const int run = blockIdx.x >> 1, kv = blockIdx.x & 1, slot = run / p.heads, rest = run - slot * p.heads;
    pdl_launch_dependents();
    pdl_wait();
    const EvictSlot s = evict_slot(a, slot);
    if (a.out_status[slot] != MTP_OK || s.after == s.len) return;
    const int* table = a.block_table + (long long)slot * a.bt_stride;
    if (rest == 0 && kv == 0) free_pages<EM_THREADS>(p, s, table);
    const int layer = rest / a.n_kv_heads, head = rest - layer * a.n_kv_heads;
    move_rows<EM_THREADS, EM_UNROLL>(p, s, table, p.list + (long long)run * p.width, reinterpret_cast<uint4*>(ev_sm), layer, head, kv, 1);
}

template <int NT, bool HELD, int UNROLL, int CTAS>
cudaError_t launch_evict(EvictArgs p, int parts, cudaStream_t s) {
    const int runs = p.a.slots * p.heads;
    size_t smem = HELD ? ring_bytes(NT, UNROLL) + (size_t)p.width * 4 : EV_BINS * 4;
    if (HELD && NT == 1024) smem = EV_SMEM;  // (one CTA an SM)
    p.smem = (int)smem;
    const cudaError_t e = ensure_kernel_smem(reinterpret_cast<const void*>(evict_kernel<NT, HELD, UNROLL, CTAS>), smem);
    return e == cudaSuccess ? launch_ex(evict_kernel<NT, HELD, UNROLL, CTAS>, dim3(runs, parts), NT, smem, s, 1, p) : e;
}

size_t evict_workspace(const mtp_cache_evict_args* a) {
    const size_t width = (size_t)a->bt_stride * a->page_size;
    return width <= EV_HELD ? 0 : (size_t)a->slots * a->layers * a->n_kv_heads * width * sizeof(int);
}
bool evict_sizes(const mtp_cache_evict_args* a) {
    return a && a->slots >= 1 && a->slots <= 8192 && a->bt_stride >= 1 && page_size_ok(a->page_size) &&
           (long long)a->bt_stride * a->page_size <= 1 << 24 && a->layers >= 1 && a->n_kv_heads >= 1 && a->n_kv_heads <= 1024 &&
           (long long)a->slots * a->layers * a->n_kv_heads <= 1 << 28;
}

}  // namespace
}  // namespace mtp

using namespace mtp;

extern "C" {

MTP_API size_t mtp_cache_evict_workspace_bytes(const mtp_cache_evict_args* a) {
    return evict_sizes(a) ? evict_workspace(a) : 0;
}

MTP_API int mtp_cache_evict(const mtp_cache_evict_args* a, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return guarded([&]() -> int {
        if (!a) return invalid("cache_evict: null arguments");
        if (const int r = check_pool("cache_evict", a->n_pages, a->layers, 0, a->n_kv_heads, a->head_dim, a->page_size)) return r;
        if (!evict_sizes(a)) return invalid("cache_evict: invalid sizes (slots %d, bt_stride %d)", a->slots, a->bt_stride);
        if (a->pool_dtype != MTP_BF16 && a->pool_dtype != MTP_F16) return invalid("cache_evict: pool_dtype %d", a->pool_dtype);
        if (a->sinks < 0 || a->recent < 0) return invalid("cache_evict: sinks %d, recent %d", a->sinks, a->recent);
        if (!a->kv_lens || !a->keep || !a->block_table || !a->page_refs || !a->weights || !a->kv_pool || !a->out_kv_lens ||
            !a->out_block_table || !a->out_page_refs || !a->out_weights || !a->out_status)
            return invalid("cache_evict: null pointer");
        if (a->out_block_table == a->block_table || a->out_kv_lens == a->kv_lens || a->out_kv_lens == a->keep ||
            a->out_weights == a->weights)
            return invalid("cache_evict: the new lengths, tables and weights need buffers of their own");
        if (!aligned16(a->kv_pool)) return invalid("cache_evict: kv_pool must be 16-byte aligned");
        if (evict_workspace(a) > 0 && (!workspace || !aligned16(workspace) || workspace_bytes < evict_workspace(a)))
            return invalid("cache_evict: workspace %zu bytes, need %zu, 16-byte aligned", workspace_bytes, evict_workspace(a));
        const EvictArgs p{*a, log2_of(a->page_size), a->bt_stride * a->page_size, a->layers * a->n_kv_heads, 0, aligned16(a->weights), static_cast<int*>(workspace)};
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        const int runs = a->slots * p.heads;
        int dev = 0, sms = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e == cudaSuccess)
            e = launch_ex(evict_check_kernel, dim3(std::max(a->slots, std::min(sms, a->n_pages / (4 * EC_THREADS)))), EC_THREADS, 0, s, 1, p);
        if (e != cudaSuccess) return cuda_status(e, "cache_evict");
        if (p.width <= EV_HELD) {
            // Threads by the table's width, whose keys shared memory holds: CTAs of an SM 5, 3, 2, 1 (and the registers that go with them: with
            // those of 3, 8 slots of up to 10,000 keys took 249 us, with those of 2 202).  Where all keys and values have room on the SMs at
            // once, a CTA each (both make the selection).  256 threads, 512: 16 slots of up to 2000 keys 136, 160 us, 24 of up to 2500 105, 115;
            // 8 of up to 3000 154, 146, of up to 4000 293, 270.
            if (p.width <= 4096 && runs * 2 <= 3 * sms)
                e = launch_evict<512, true, 1, 3>(p, 2, s);
            else if (p.width <= 2816)
                e = launch_evict<256, true, 2, 5>(p, 1, s);
            else if (p.width <= 12288)
                e = launch_evict<512, true, 1, 2>(p, runs * 2 <= 2 * sms ? 2 : 1, s);
            else
                e = launch_evict<1024, true, 1, 1>(p, runs * 2 <= sms ? 2 : 1, s);
        } else {
            e = launch_evict<1024, false, 1, 1>(p, 1, s);
            if (e == cudaSuccess) e = launch(evict_move_kernel, runs * 2, EM_THREADS, ring_bytes(EM_THREADS, EM_UNROLL), 1, s, p);
        }
        return cuda_status(e, "cache_evict");
    });
}

}  // extern "C"
