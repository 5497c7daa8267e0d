// evict.cu -- contexts brought down to a budget of keys (mtp_cache_evict): of every slot, layer and
// key head the keys of largest weight stay, beside the first and the last ones, move up in their
// order, and the pages behind them become free.
//
// Two kernels.  The first selects: a CTA has the weights of one (slot, layer, key head) in registers, as
// whole numbers in the order of the weights, and finds the m-th largest bit by bit, each
// bit with one count over the CTA (no atomics, and nothing depends on how weights are spread).  Of the keys
// equal to it the first ones stay.  Ballots and prefix sums then give each key that stays its place; its
// row in the pool goes to a list in the workspace.
// The second moves keys and values in place: a CTA has one (slot, layer, key head, keys | values) run and
// goes through its list from the front, a block of rows at a time: read, barrier, write.  Row j is
// read from place old_j >= j, and rows before a block's are never read again, so that no copy of the
// cache is needed; the next block is read before this one is written.
#include <algorithm>
#include <climits>

#include "serving.cuh"

namespace mtp {
namespace {

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

template <int NT, int KPT>
__global__ void __launch_bounds__(NT) evict_select_kernel(const __grid_constant__ EvictArgs p) {
    constexpr int WARPS = NT / 32, TILE = NT * KPT;
    __shared__ uint32_t count[2][WARPS], lows[WARPS], ties_of[WARPS], kept_of[WARPS];
    const mtp_cache_evict_args& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int run = blockIdx.x, slot = run / p.heads, first_run = run - slot * p.heads == 0;
    pdl_launch_dependents();
    pdl_wait();
    const int mask = (1 << p.shift) - 1;
    if (a.out_page_refs != a.page_refs)
        for (long long i = (long long)run * NT + tid; i < a.n_pages; i += (long long)gridDim.x * NT) a.out_page_refs[i] = a.page_refs[i];
    const EvictSlot s = evict_slot(a, slot);
    const int* table = a.block_table + (long long)slot * a.bt_stride;
    bool bad = s.len < 0 || s.len > p.width || a.keep[slot] < 0;
    if (!bad && s.after < s.len) {
        // every held page is one and is counted; those that are written are in no other table
        const int held = (s.len + mask) >> p.shift, written = (s.after + mask) >> p.shift, same = s.sinks >> p.shift;
        for (int c = tid; c < held; c += NT) {
            const int page = table[c], n = page >= 0 && page < a.n_pages ? a.page_refs[page] : 0;
            bad |= n < 1 || (n > 1 && c >= same && c < written);
        }
    }
    bad = __syncthreads_or(bad) != 0;
    if (first_run) {
        const int left = bad || s.after == s.len ? a.bt_stride : (s.after + mask) >> p.shift;
        for (int c = tid; c < a.bt_stride; c += NT) {
            const bool unused = !bad && c >= (s.after + mask) >> p.shift;
            a.out_block_table[(long long)slot * a.bt_stride + c] = unused || c >= left ? -1 : table[c];
        }
        if (tid == 0) {
            a.out_kv_lens[slot] = bad ? s.len : s.after;
            a.out_status[slot] = bad ? MTP_ERR_INVALID : MTP_OK;
        }
    }
    const float* w = a.weights + (long long)run * p.width;
    float* out = a.out_weights + (long long)run * p.width;
    if (bad || s.after == s.len) {  // nothing moves
        for (int i = tid; i < min(max(s.len, 0), p.width); i += NT) out[i] = w[i];
        return;
    }
    const int lo = s.sinks, hi = s.len - s.recent, want = s.after - s.sinks - s.recent;  // of keys [lo, hi) so many
    uint32_t key[KPT];
    const int tiles = (s.len + TILE - 1) / TILE;
    auto load = [&](int tile) {  // key i of a thread: 32 consecutive ones of the warp's part of the tile
        const int base = tile * TILE + warp * (32 * KPT) + lane;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const int at = base + i * 32;
            key[i] = at >= lo && at < hi ? order_of(w[at]) : 0u;
        }
    };
    load(0);
    // the want-th largest: bits from the highest in which the keys differ
    uint32_t high = 0, low = 0xffffffffu;
    for (int t = 0; t < tiles; ++t) {
        if (t > 0) load(t);
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            high = max(high, key[i]);
            low = min(low, key[i] - 1);  // (0: none)
        }
    }
    high = __reduce_max_sync(FULL_MASK, high);
    low = __reduce_min_sync(FULL_MASK, low);
    if (lane == 0) {
        count[0][warp] = high;
        lows[warp] = low;
    }
    __syncthreads();
    high = __reduce_max_sync(FULL_MASK, lane < WARPS ? count[0][lane] : 0u);
    low = __reduce_min_sync(FULL_MASK, lane < WARPS ? lows[lane] : 0xffffffffu) + 1;
    uint32_t border = want > 0 ? low : 0xffffffffu;
    if (want > 0 && low != high) {
        const int top = 31 - __clz(low ^ high);
        border = low & ~((2u << top) - 1);
        if (top == 31) border = 0;
        int turn = 1;
        for (int bit = top; bit >= 0; --bit) {
            const uint32_t next = border | 1u << bit;
            uint32_t n = 0;
            for (int t = 0; t < tiles; ++t) {
                if (tiles > 1) load(t);
#pragma unroll
                for (int i = 0; i < KPT; ++i) n += key[i] >= next;
            }
            n = __reduce_add_sync(FULL_MASK, n);
            if (lane == 0) count[turn][warp] = n;
            __syncthreads();
            n = __reduce_add_sync(FULL_MASK, lane < WARPS ? count[turn][lane] : 0u);
            turn ^= 1;
            if (n >= (uint32_t)want) border = next;
            if (n == (uint32_t)want) break;
        }
    }
    // how many above the border, of those on it the first ones; then every kept key's place
    int ties_left = want, place = 0;  // of the tiles before
    for (int pass = 0; pass < 2; ++pass) {
        if (pass == 0) {  // the number above the border
            uint32_t n = 0;
            for (int t = 0; t < tiles; ++t) {
                if (tiles > 1) load(t);
#pragma unroll
                for (int i = 0; i < KPT; ++i) n += want > 0 && key[i] > border;
            }
            n = __reduce_add_sync(FULL_MASK, n);
            __syncthreads();
            if (lane == 0) lows[warp] = n;
            __syncthreads();
            ties_left -= (int)__reduce_add_sync(FULL_MASK, lane < WARPS ? lows[lane] : 0u);
            continue;
        }
        for (int t = 0; t < tiles; ++t) {
            if (tiles > 1) load(t);
            const int base = t * TILE + warp * (32 * KPT) + lane;
            auto forced = [&](int at) { return at < lo || (at >= hi && at < s.len); };
            int ties = 0, sure = 0;
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                ties += __popc(__ballot_sync(FULL_MASK, want > 0 && key[i] == border));
                sure += __popc(__ballot_sync(FULL_MASK, (want > 0 && key[i] > border) || forced(base + i * 32)));
            }
            __syncthreads();  // (the tile before is still read)
            if (lane == 0) {
                ties_of[warp] = ties;
                kept_of[warp] = sure;
            }
            __syncthreads();
            const int x = lane < WARPS ? (int)ties_of[lane] : 0, y = lane < WARPS ? (int)kept_of[lane] : 0;
            const int ties_before = __reduce_add_sync(FULL_MASK, lane < warp ? x : 0), ties_all = __reduce_add_sync(FULL_MASK, x);
            int to = place + __reduce_add_sync(FULL_MASK, lane < warp ? y : 0) + min(ties_before, ties_left);
            int left = max(0, ties_left - ties_before);
            place += __reduce_add_sync(FULL_MASK, y) + min(ties_all, ties_left);
            ties_left = max(0, ties_left - ties_all);
            const unsigned below = (1u << lane) - 1;
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                const int at = base + i * 32;
                const bool tie = want > 0 && key[i] == border;
                const unsigned tied = __ballot_sync(FULL_MASK, tie);
                const bool keep = (want > 0 && key[i] > border) || forced(at) || (tie && __popc(tied & below) < left);
                const unsigned kept = __ballot_sync(FULL_MASK, keep);
                if (keep) {
                    const int dst = to + __popc(kept & below);
                    out[dst] = w[at];
                    p.list[(long long)run * p.width + dst] = (table[at >> p.shift] << p.shift) + (at & mask);
                }
                to += __popc(kept);
                left = max(0, left - __popc(tied));
            }
        }
    }
}

constexpr int EV_THREADS = 256, EV_UNROLL = 4;

// Grid (run * 2 + keys | values).
__global__ void __launch_bounds__(EV_THREADS) evict_move_kernel(const __grid_constant__ EvictArgs p) {
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
    const unsigned vecs = a.head_dim / 8, total = (unsigned)(s.after - s.sinks) * vecs;
    const int* list = p.list + (long long)run * p.width + s.sinks;
    uint4* pool = static_cast<uint4*>(a.kv_pool);
    // piece v of row `row` of the pool (page * page_size + offset)
    auto at = [&](int row, unsigned v) {
        const long long block = (((long long)(row >> p.shift) * a.layers + layer) * 2 + kv) * a.n_kv_heads + head;
        return pool + ((block << p.shift) + (row & mask)) * vecs + v;
    };
    struct Block {
        uint4 x[EV_UNROLL];
        uint4* to[EV_UNROLL];
    };
    auto read = [&](Block& b, unsigned i0) {
#pragma unroll
        for (int u = 0; u < EV_UNROLL; ++u) {
            const unsigned i = i0 + u * EV_THREADS + tid;
            b.to[u] = nullptr;
            if (i >= total) continue;
            const unsigned j = i / vecs, v = i - j * vecs;
            const int from = list[j], now = (int)j + s.sinks, to = (table[now >> p.shift] << p.shift) + (now & mask);
            if (from == to) continue;
            b.x[u] = *at(from, v);
            b.to[u] = at(to, v);
        }
    };
    auto write = [&](const Block& b) {
#pragma unroll
        for (int u = 0; u < EV_UNROLL; ++u)
            if (b.to[u]) *b.to[u] = b.x[u];
    };
    constexpr unsigned STEP = EV_THREADS * EV_UNROLL;
    Block x, y;
    read(x, 0);
    for (unsigned i = 0; i < total; i += 2 * STEP) {
        read(y, i + STEP);
        __syncthreads();  // every row of this block and the next is read
        write(x);
        read(x, i + 2 * STEP);
        __syncthreads();
        write(y);
    }
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
        if (p.width <= 2048)
            e = launch_ex(evict_select_kernel<256, 8>, dim3(runs), 256, 0, s, 1, p);
        else if (p.width <= 8192)
            e = launch_ex(evict_select_kernel<512, 16>, dim3(runs), 512, 0, s, 1, p);
        else
            e = launch_ex(evict_select_kernel<512, 64>, dim3(runs), 512, 0, s, 1, p);
        if (e == cudaSuccess) e = launch_ex(evict_move_kernel, dim3(runs * 2), EV_THREADS, 0, s, 1, p);
        return cuda_status(e, "cache_evict");
    });
}

}  // extern "C"
