// evict.cu -- contexts brought down to a budget of keys (mtp_cache_evict): of every slot, layer and
// key head the keys of largest weight stay, beside the first and the last ones, move up in their
// order, and the pages behind them become free.
//
// Two kernels.  The first selects: a CTA has the weights of one (slot, layer, key head) in shared memory, as
// whole numbers in the order of the weights, and finds the m-th largest by its highest 11 bits, the 11
// after them and the last 10, each time by counting how many keys have each value.  Of the keys
// equal to it the first ones stay.  Ballots and prefix sums then give each key that stays its place; its
// row in the pool goes to a list in the workspace.
// The second moves keys and values in place: a CTA has one (slot, layer, key head, keys | values) run and
// goes through its list from the front, a stage of rows at a time: read, barrier, write.  Row j is
// read from place old_j >= j, and places before a stage's are never read again, so that no copy of the
// cache is needed; further stages are on their way into shared memory meanwhile.
#include <algorithm>
#include <climits>

#include "serving.cuh"

namespace mtp {
namespace {

constexpr int EV_BINS = 2048;
constexpr int EV_HELD = 53248;  // keys whose order shared memory holds

struct EvictArgs {
    mtp_cache_evict_args a;
    int shift;      // page_size = 1 << shift
    int width;      // bt_stride * page_size: weights of a slot, layer and head
    int heads;      // layers * n_kv_heads
    int* list;      // workspace [slots][layers][heads][width]: row of the pool (page * page_size + offset) of each key that stays
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

// HELD: the weights' order is kept in shared memory; else (rows past EV_HELD keys) it is made again in every pass.
template <int NT, bool HELD>
__global__ void __launch_bounds__(NT) evict_select_kernel(const __grid_constant__ EvictArgs p) {
    constexpr int WARPS = NT / 32, B = EV_BINS / NT;
    extern __shared__ uint32_t ev_keys[];  // [width]
    __shared__ __align__(16) uint32_t bins[EV_BINS];
    __shared__ uint32_t part[WARPS], tied_of[WARPS], kept_of[WARPS];
    __shared__ int s_bin, s_left, s_count;
    const mtp_cache_evict_args& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int run = blockIdx.x, slot = run / p.heads;
    const bool first_run = run - slot * p.heads == 0;
    pdl_launch_dependents();
    for (int i = tid; i < EV_BINS; i += NT) bins[i] = 0;
    pdl_wait();
    const int mask = (1 << p.shift) - 1;
    const EvictSlot s = evict_slot(a, slot);
    const float* w = a.weights + (long long)run * p.width;
    const int lo = s.sinks, hi = s.len - s.recent, want = s.after - s.sinks - s.recent;  // of keys [lo, hi) so many
    bool bad = s.len < 0 || s.len > p.width || a.keep[slot] < 0;
    if (a.out_page_refs != a.page_refs)
        for (long long i = (long long)run * NT + tid; i < a.n_pages; i += (long long)gridDim.x * NT) a.out_page_refs[i] = a.page_refs[i];
    const int* table = a.block_table + (long long)slot * a.bt_stride;
    const bool moves = !bad && s.after < s.len;
    auto order_at = [&](int at) { return at >= lo && at < hi ? order_of(w[at]) : 0u; };  // 0: not to be chosen
    if (moves) {
        // every held page is one and is counted; those that are written are in no other table
        const int held = (s.len + mask) >> p.shift, written = (s.after + mask) >> p.shift, same = s.sinks >> p.shift;
        int page[2];
        auto look = [&](int c) { return c < held ? table[c] : INT_MAX; };
        page[0] = look(tid);
        page[1] = look(tid + NT);
        if (HELD)
#pragma unroll 8
            for (int i = tid; i < s.len; i += NT) ev_keys[i] = order_at(i);
        for (int c = tid; c < held; c += 2 * NT) {
            int n[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) n[e] = page[e] >= 0 && page[e] < a.n_pages ? a.page_refs[page[e]] : 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int at = c + e * NT;
                bad |= at < held && (n[e] < 1 || (n[e] > 1 && at >= same && at < written));
                page[e] = look(at + 2 * NT);
            }
        }
    }
    bad = __syncthreads_or(bad) != 0;
    if (first_run) {
        const int used = bad ? a.bt_stride : (s.after + mask) >> p.shift;
        for (int c = tid; c < a.bt_stride; c += NT) a.out_block_table[(long long)slot * a.bt_stride + c] = c < used ? table[c] : -1;
        if (tid == 0) {
            a.out_kv_lens[slot] = bad ? s.len : s.after;
            a.out_status[slot] = bad ? MTP_ERR_INVALID : MTP_OK;
        }
    }
    float* out = a.out_weights + (long long)run * p.width;
    if (bad || !moves) {
        for (int i = tid; i < min(max(s.len, 0), p.width); i += NT) out[i] = w[i];
        return;
    }
    auto key_at = [&](int at) { return at >= s.len ? 0u : HELD ? ev_keys[at] : order_at(at); };

    // the want-th largest, from its highest bits: how many keys have each value of the next 11 bits
    uint32_t border = 0;
    int left = want;   // keys that stay of those on the border
    bool all = false;  // all of those on the border stay
    if (want > 0)
#pragma unroll 1
        for (int shift = 21, width = 11; !all;) {
#pragma unroll 4
            for (int i0 = warp * 32; i0 < s.len; i0 += NT) {
                const uint32_t key = key_at(i0 + lane);
                const bool in = key != 0 && (shift == 21 || (key ^ border) >> (shift + width) == 0);
                const unsigned who = __ballot_sync(FULL_MASK, in);
                if (who == 0) continue;
                // a warp's keys that are all alike are one addition (weights that are all 0, say)
                const uint32_t digit = key >> shift & ((1u << width) - 1);
                const int leader = __ffs(who) - 1;
                const uint32_t first = __shfl_sync(FULL_MASK, digit, leader);
                if (__all_sync(FULL_MASK, !in || digit == first)) {
                    if (lane == leader) atomicAdd(&bins[digit], __popc(who));
                } else if (in) {
                    atomicAdd(&bins[digit], 1u);
                }
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
            width = shift == 21 ? 11 : 10;
            shift -= width;
        }
    // a warp's keys, in their order: how many stay for sure, and how many are on a border of which only the first `left` stay
    const int per = ((s.len + NT - 1) / NT) * 32, first = warp * per, last = min(s.len, first + per);
    const bool ties = want > 0 && !all;
    border = want > 0 ? max(border, 1u) : 0xffffffffu;
    auto sure = [&](int at, uint32_t key) {
        return at < lo || (at >= hi && at < s.len) || (want > 0 && (ties ? key > border : key >= border));
    };
    int n_sure = 0, n_tied = 0;
#pragma unroll 4
    for (int i0 = first; i0 < last; i0 += 32) {
        const int at = i0 + lane;
        const uint32_t key = key_at(at);
        n_sure += __popc(__ballot_sync(FULL_MASK, sure(at, key)));
        if (ties) n_tied += __popc(__ballot_sync(FULL_MASK, key == border));
    }
    if (lane == 0) {
        kept_of[warp] = n_sure;
        tied_of[warp] = n_tied;
    }
    __syncthreads();
    const int tied_before = (int)__reduce_add_sync(FULL_MASK, lane < warp ? tied_of[lane] : 0u);
    int place = (int)__reduce_add_sync(FULL_MASK, lane < warp ? kept_of[lane] : 0u) + (ties ? min(tied_before, left) : 0);
    left = max(0, left - tied_before);
    int* list = p.list + (long long)run * p.width;
    const unsigned below = (1u << lane) - 1;
    constexpr int BATCH = 4;  // whose reads are on their way together
    for (int i0 = first; i0 < last; i0 += 32 * BATCH) {
        int dst[BATCH], page[BATCH];
        float weight[BATCH];
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            const int at = i0 + e * 32 + lane;
            const bool there = at < last;
            const uint32_t key = there ? key_at(at) : 0u;
            bool keep = there && sure(at, key);
            if (ties) {
                const unsigned tied = __ballot_sync(FULL_MASK, key == border);
                keep |= key == border && __popc(tied & below) < left;
                left = max(0, left - __popc(tied));
            }
            const unsigned kept = __ballot_sync(FULL_MASK, keep);
            dst[e] = keep ? place + __popc(kept & below) : -1;
            place += __popc(kept);
            page[e] = keep ? table[at >> p.shift] : 0;
            // the weight is in its order but for the sign of 0 and NaN's bits, and where there is none
            const bool plain = key != 0 && key != 0x80000000u && key != 0xffffffffu;
            weight[e] = plain ? __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key) : keep ? w[at] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < BATCH; ++e) {
            if (dst[e] < 0) continue;
            out[dst[e]] = weight[e];
            list[dst[e]] = (page[e] << p.shift) + ((i0 + e * 32 + lane) & mask);
        }
    }
}

constexpr int EV_THREADS = 256, EV_STAGES = 6;

__device__ __forceinline__ void copy16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(dst)), "l"(src) : "memory");
}

// Grid (run * 2 + keys | values).  A thread has a fixed 16-byte piece of a row, in every EV_UNROLL * (threads / pieces)-th row; it
// writes what it has read itself, so that the stages need no barrier of their own.
template <int EV_UNROLL>
__global__ void __launch_bounds__(EV_THREADS) evict_move_kernel(const __grid_constant__ EvictArgs p) {
    extern __shared__ uint4 ev_ring[];  // [EV_STAGES][EV_UNROLL][EV_THREADS]
    const mtp_cache_evict_args& a = p.a;
    const int tid = threadIdx.x, run = blockIdx.x >> 1, kv = blockIdx.x & 1, slot = run / p.heads, rest = run - slot * p.heads;
    pdl_launch_dependents();
    pdl_wait();
    const EvictSlot s = evict_slot(a, slot);
    if (a.out_status[slot] != MTP_OK || s.after == s.len) return;
    const int* table = a.block_table + (long long)slot * a.bt_stride;
    const int mask = (1 << p.shift) - 1;
    if (rest == 0 && kv == 0)  // the slot's pages that become free
        for (int c = ((s.after + mask) >> p.shift) + tid; c < (s.len + mask) >> p.shift; c += EV_THREADS) atomicSub(a.out_page_refs + table[c], 1);
    const int layer = rest / a.n_kv_heads, head = rest - layer * a.n_kv_heads;
    const int vecs = a.head_dim / 8, rows = EV_THREADS / vecs, r0 = tid / vecs, v = tid - r0 * vecs, step = rows * EV_UNROLL;
    const bool active = r0 < rows;
    const int* list = p.list + (long long)run * p.width;
    // a piece of row `row` (page * page_size + offset): the pool's blocks of a page apart, the head's among them
    uint4* pool = static_cast<uint4*>(a.kv_pool) + ((((long long)layer * 2 + kv) * a.n_kv_heads + head) << p.shift) * vecs + v;
    const long long page_step = ((long long)p.heads * 2 << p.shift) * vecs;
    auto at = [&](int page, int offset) { return pool + page * page_step + offset * vecs; };
    int from[EV_UNROLL];  // rows of the stage that is asked for next, on their way
    auto look = [&](int j0) {
#pragma unroll
        for (int u = 0; u < EV_UNROLL; ++u) {
            const int j = j0 + u * rows + r0;
            from[u] = active && j < s.after ? list[j] : -1;
        }
    };
    auto ask = [&](int stage) {
#pragma unroll
        for (int u = 0; u < EV_UNROLL; ++u)
            if (from[u] >= 0) copy16(ev_ring + (stage * EV_UNROLL + u) * EV_THREADS + tid, at(from[u] >> p.shift, from[u] & mask));
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
        asm volatile("cp.async.wait_group %0;" ::"n"(EV_STAGES - 2) : "memory");
        __syncthreads();  // every row of this stage and the ones before is read
        ask(in);
        look(next += step);
#pragma unroll
        for (int u = 0; u < EV_UNROLL; ++u) {
            const int j = j0 + u * rows + r0;
            if (active && j < s.after) *at(table[j >> p.shift], j & mask) = ev_ring[(out * EV_UNROLL + u) * EV_THREADS + tid];
        }
        in = in + 1 == EV_STAGES ? 0 : in + 1;
        out = out + 1 == EV_STAGES ? 0 : out + 1;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

template <int UNROLL>
cudaError_t launch_move(const EvictArgs& p, int ctas, cudaStream_t s) {
    return launch(evict_move_kernel<UNROLL>, ctas, EV_THREADS, (size_t)EV_STAGES * UNROLL * EV_THREADS * 16, 1, s, p);
}
cudaError_t launch_move(const EvictArgs& p, int ctas, cudaStream_t s) {
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    return ctas > 2 * sms ? launch_move<2>(p, ctas, s) : launch_move<4>(p, ctas, s);
}

size_t evict_workspace(const mtp_cache_evict_args* a) {
    return (size_t)a->slots * a->layers * a->n_kv_heads * a->bt_stride * a->page_size * sizeof(int);
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
        if (!workspace || !aligned16(workspace) || workspace_bytes < evict_workspace(a))
            return invalid("cache_evict: workspace %zu bytes, need %zu, 16-byte aligned", workspace_bytes, evict_workspace(a));
        const EvictArgs p{*a, log2_of(a->page_size), a->bt_stride * a->page_size, a->layers * a->n_kv_heads, static_cast<int*>(workspace)};
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        const int runs = a->slots * p.heads;
        cudaError_t e;
        const size_t held = p.width <= EV_HELD ? (size_t)p.width * sizeof(uint32_t) : 0;
        if (p.width <= 4096)
            e = launch(evict_select_kernel<256, true>, runs, 256, held, 1, s, p);
        else if (held > 0)
            e = launch(evict_select_kernel<1024, true>, runs, 1024, held, 1, s, p);
        else
            e = launch(evict_select_kernel<1024, false>, runs, 1024, 0, 1, s, p);
        if (e == cudaSuccess) e = launch_move(p, runs * 2, s);
        return cuda_status(e, "cache_evict");
    });
}

}  // extern "C"
