// paged.cu -- the paged cache's bookkeeping on the GPU: pages, block tables and
// slot maps of a step's new tokens (mtp_page_plan), the new keys and values into
// the cache (mtp_cache_append), and the cache of the beams that a selection keeps
// (mtp_beam_reorder).
//
// A page is free where its count is zero.  Pages are taken lowest number first,
// in the order of the requests, so the outcome does not depend on how the work is
// spread: with f_0 < f_1 < ... the free pages and need(s) the pages that request s
// lacks, request s takes f_{N(s)} .. f_{N(s) + need(s) - 1}, N(s) = sum_{s' < s} need(s').
// Both sides are prefix sums: over the requests (every CTA makes the whole one, in
// shared memory), and over the counts, of which each of the cluster's CTAs reads a
// part once and keeps a bit per page; CTA totals go over distributed shared memory.
// A free page then finds its request by a binary search of its rank.
//
// What bounds them is latency: a handful of dependent steps with a barrier between them (the
// ranks before the tables, the tables before the rows that look pages up).  One CTA does a
// serving step's work; where there are more pages, requests or tables than its threads
// get through in a step, a cluster of eight (a barrier of the cluster takes about a
// microsecond, one of a CTA a few dozen cycles, a second launch more than either).  The plan's
// rows, of which a prompt batch has hundreds of thousands, are then written by the whole
// GPU in a launch of their own.
// Times of calls, one after another: plan of 32 slots, one token each, 2048 pages 3.8 us; of 1000
// slots, 300,000 rows, 90,001 pages 21.3 us (5 MB written: the chain of steps, most of all the
// taking of 10,000 pages by eight CTAs); reordering of 4 beams 8.2 us, of 96 beams, 36 of them copied,
// with 12 layers of 16 heads of 64 21.2 us.
#include <climits>

#include "serving.cuh"

namespace mtp {
namespace {

constexpr int PG_CLUSTER = 8, PG_THREADS = 1024, PG_WARPS = PG_THREADS / 32;
// One CTA up to these.  One CTA against eight, us a call: plan of 32 slots and 2048 pages 3.9 and 4.9, 8192 pages 4.4 and 5.0,
// 16384 pages 5.5 and 5.1, 32768 pages 7.5 and 5.2; of 1024 slots and 34,000 pages 9.6 and 7.2; 2048 rows beside them 6.5 and 5.7;
// reordering of 96 beams 10.3 and 12.7, of 256 beams 13.7 and 12.8, of 512 19.1 and 14.0.
constexpr int PG_ONE_PAGES = 8192, PG_ONE_SLOTS = 1024, PG_ONE_ROWS = 1024, PG_ONE_BEAMS = 192;
// Rows that the plan's own launch writes, more are written by one of theirs: 4096 rows 5.7 and 8.9 us, 8192 5.9 and 9.4, 16384
// 6.5 and 8.9.
constexpr int PG_ROWS_HERE = 16384;
constexpr int PG_MAX_SLOTS = 8192;
constexpr int PG_MAX_ROWS = 1 << 24;

struct FreeBits {
    uint32_t* bits;       // shared memory: a bit per page of this CTA's part, set where it is free
    uint32_t* before;     // [words] free pages of the part before each word
    int first, words;     // the part: words [first, first + words) of 32 pages
};

__host__ __device__ inline int free_words(int n_pages, int ctas) {  // words of a CTA's part
    return ((n_pages + 31) / 32 + ctas - 1) / ctas;
}

// Exclusive prefix sum of x over the block and the total, both below 2^32.  Synchronises the block.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* part, uint32_t& sum) {
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
    const uint32_t mine = part[lane];
    sum = __reduce_add_sync(FULL_MASK, mine);
    return __reduce_add_sync(FULL_MASK, lane < warp ? mine : 0) + y - x;
}

// The same of two numbers, and the sum alone of a third, between the same barriers.
struct ScanParts {
    uint32_t x[PG_WARPS], y[PG_WARPS], z[PG_WARPS];
};
__device__ __forceinline__ void block_scan3(uint32_t& x, uint32_t& y, uint32_t z, ScanParts& part, uint32_t& sum_x, uint32_t& sum_y,
                                            uint32_t& sum_z) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t u = x, v = y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t p = __shfl_up_sync(FULL_MASK, u, o), q = __shfl_up_sync(FULL_MASK, v, o);
        if (lane >= o) {
            u += p;
            v += q;
        }
    }
    z = __reduce_add_sync(FULL_MASK, z);
    __syncthreads();
    if (lane == 31) {
        part.x[warp] = u;
        part.y[warp] = v;
        part.z[warp] = z;
    }
    __syncthreads();
    const uint32_t p = part.x[lane], q = part.y[lane];
    sum_x = __reduce_add_sync(FULL_MASK, p);
    sum_y = __reduce_add_sync(FULL_MASK, q);
    sum_z = __reduce_add_sync(FULL_MASK, part.z[lane]);
    x = __reduce_add_sync(FULL_MASK, lane < warp ? p : 0) + u - x;
    y = __reduce_add_sync(FULL_MASK, lane < warp ? q : 0) + v - y;
}

// Reads this CTA's part of the counts once (and copies it, where they go to another
// array); leaves the part's free pages in *total.
template <int CTAS>
__device__ __forceinline__ FreeBits find_free(const int* refs, int* out_refs, int n_pages, int rank, uint32_t* bits,
                                              uint32_t* part, int* total) {
    constexpr int UNROLL = 8;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    FreeBits f;
    const int all = (n_pages + 31) / 32, cap = free_words(n_pages, CTAS);
    f.bits = bits;
    f.before = bits + cap;
    f.first = rank * cap;
    f.words = max(0, min(cap, all - f.first));
    const bool copy = out_refs != refs;
    for (int w0 = warp; w0 < f.words; w0 += PG_WARPS * UNROLL) {
        int r[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int w = w0 + u * PG_WARPS, i = (f.first + w) * 32 + lane;
            r[u] = w < f.words && i < n_pages ? refs[i] : 1;
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int w = w0 + u * PG_WARPS, i = (f.first + w) * 32 + lane;
            if (w >= f.words) break;
            const unsigned b = __ballot_sync(FULL_MASK, r[u] == 0);
            if (copy && i < n_pages) out_refs[i] = r[u];
            if (lane == 0) bits[w] = b;
        }
    }
    __syncthreads();
    const int per = (f.words + PG_THREADS - 1) / PG_THREADS;  // words of a thread, consecutive
    uint32_t n = 0, sum;
    for (int w = tid * per; w < min((tid + 1) * per, f.words); ++w) n += __popc(bits[w]);
    n = block_scan(n, part, sum);
    for (int w = tid * per; w < min((tid + 1) * per, f.words); ++w) {
        f.before[w] = n;
        n += __popc(bits[w]);
    }
    if (tid == 0) *total = (int)sum;
    return f;
}

// take(page, rank) for the free pages of this CTA's part whose rank among all is below `want`: a
// warp takes a word of the bits at a time, a lane a page.
template <class F>
__device__ __forceinline__ void take_free(const FreeBits& f, long long base, long long want, F take) {
    const int lane = threadIdx.x & 31;
    for (int w = threadIdx.x >> 5; w < f.words; w += PG_WARPS) {
        const long long first = base + f.before[w];
        if (first >= want) break;
        const uint32_t b = f.bits[w];
        const long long rank = first + __popc(b & ((1u << lane) - 1));
        if ((b >> lane & 1) && rank < want) take((f.first + w) * 32 + lane, (int)rank);
    }
}

__device__ __forceinline__ int ld_dsmem_int(const int* p, int rank) {
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(dsmem_addr(p, rank)) : "memory");
    return v;
}
// A barrier of the CTAs that work together, after which they see each other's writes; with its two halves apart.
template <int CTAS>
__device__ __forceinline__ void team_arrive() {
    if constexpr (CTAS > 1) cluster_arrive_release();
}
template <int CTAS>
__device__ __forceinline__ void team_wait() {
    if constexpr (CTAS == 1) __syncthreads(); else cluster_wait();
}
template <int CTAS>
__device__ __forceinline__ void team_barrier() {
    team_arrive<CTAS>();
    team_wait<CTAS>();
}
// Sum of a shared-memory word of every CTA; *before: of those below `rank`.
template <int CTAS>
__device__ __forceinline__ long long team_sum(const int* word, int rank, long long* before) {
    long long all = 0, low = 0;
#pragma unroll
    for (int c = 0; c < CTAS; ++c) {
        const int n = CTAS == 1 ? *word : ld_dsmem_int(word, c);
        if (c < rank) low += n;
        all += n;
    }
    if (before) *before = low;
    return all;
}

// largest s in [0, n) with before[s] <= x (before ascending, before[0] = 0 <= x)
__device__ __forceinline__ int owner_of(const int* before, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int pages_of(int tokens, int shift) { return (tokens + (1 << shift) - 1) >> shift; }

struct PlanRow {
    int64_t at;
    int seq, pos;
};
// Row r of the plan: its slot, position and place; none (-1) past the last.
__device__ __forceinline__ PlanRow plan_row(int r, int rows, const int* before, const int* lens, int slots,
                                            const int* table, int stride, int n_pages, int shift) {
    PlanRow o{-1, -1, -1};
    if (r >= rows) return o;
    o.seq = owner_of(before, slots, r);
    o.pos = lens[o.seq] + r - before[o.seq];
    const int page = __ldcg(table + (size_t)o.seq * stride + (o.pos >> shift));
    if (page >= 0 && page < n_pages) o.at = ((int64_t)page << shift) + (o.pos & ((1 << shift) - 1));
    return o;
}

struct PlanArgs {
    mtp_page_plan_args a;
    int shift;      // page_size = 1 << shift
    int rows_here;  // write the rows in this launch
};

template <int CTAS>
__global__ void __launch_bounds__(PG_THREADS, 1) page_plan_kernel(const __grid_constant__ PlanArgs p) {
    extern __shared__ int pg_sm[];
    __shared__ uint32_t part[PG_WARPS];
    __shared__ ScanParts parts;
    __shared__ int s_free;
    const mtp_page_plan_args& a = p.a;
    const int tid = threadIdx.x, rank = CTAS == 1 ? 0 : blockIdx.x, slots = a.slots;
    int* rows_before = pg_sm;                     // [slots + 1]
    int* pages_before = rows_before + slots + 1;  // [slots + 1]
    int* lens = pages_before + slots + 1;         // [slots]
    uint32_t* bits = reinterpret_cast<uint32_t*>(lens + slots);
    pdl_launch_dependents();
    pdl_wait();

    // the first requests are on their way while the free pages are looked for, and CTAs' totals while the requests are summed
    int len = tid < slots ? a.kv_lens[tid] : 0, add = tid < slots ? a.new_lens[tid] : 0;
    const FreeBits f = find_free<CTAS>(a.page_refs, a.out_page_refs, a.n_pages, rank, bits, part, &s_free);
    team_arrive<CTAS>();

    // the requests: every CTA makes the whole prefix sums
    uint32_t rows = 0, want = 0;
    bool bad = false;
    for (int s0 = 0; s0 < slots; s0 += PG_THREADS) {
        const int s = s0 + tid;
        uint32_t x = 0, y = 0, sx, sy, thousands;
        if (s < slots) {
            if (s0 > 0) {
                len = a.kv_lens[s];
                add = a.new_lens[s];
            }
            const bool wrong = len < 0 || add < 0 || add > a.max_rows || (long long)len + add > (long long)a.bt_stride << p.shift;
            bad |= wrong;
            lens[s] = len;
            if (!wrong) {
                x = add;
                y = pages_of(len + add, p.shift) - pages_of(len, p.shift);
            }
        }
        block_scan3(x, y, x >> 12, parts, sx, sy, thousands);
        if (s < slots) {  // (more rows than 32 bits hold: nothing of this is used)
            rows_before[s] = (int)(rows + x);
            pages_before[s] = (int)(want + y);
        }
        // 1024 requests of 2^24 rows at most: where their multiples of 4096 alone are more than 2^24, their sum may have
        // passed 32 bits, and is too much in any case
        bad |= thousands > (uint32_t)PG_MAX_ROWS >> 12 || rows + sx > (uint32_t)a.max_rows;
        rows += sx;
        want += sy;
    }
    if (tid == 0) {
        rows_before[slots] = (int)rows;
        pages_before[slots] = (int)want;
    }
    int code = __syncthreads_or(bad) ? MTP_ERR_INVALID : MTP_OK;
    team_wait<CTAS>();
    long long base;
    const long long free_all = team_sum<CTAS>(&s_free, rank, &base);
    if (code == MTP_OK && want > free_all) code = MTP_ERR_NO_PAGES;
    if (code != MTP_OK) rows = want = 0;
    take_free(f, base, want, [&](int page, int n) {
        const int s = owner_of(pages_before, slots, n);
        a.block_table[(size_t)s * a.bt_stride + pages_of(lens[s], p.shift) + n - pages_before[s]] = page;
        a.out_page_refs[page] = 1;
    });
    team_barrier<CTAS>();  // the tables are written

    const int gid = rank * PG_THREADS + tid;
    for (int s = gid; s <= slots; s += CTAS * PG_THREADS) {
        const int before = code == MTP_OK ? rows_before[s] : 0;
        a.out_cu_rows[s] = before;
        if (s < slots) a.out_kv_lens[s] = code == MTP_OK ? lens[s] + rows_before[s + 1] - before : lens[s];
    }
    if (gid == 0) {
        a.out_status[0] = code;
        a.out_status[1] = (int)rows;
        a.out_status[2] = (int)want;
        a.out_status[3] = (int)(free_all - want);
    }
    if (!p.rows_here) return;
    for (int r = gid; r < a.max_rows; r += CTAS * PG_THREADS) {
        const PlanRow o = plan_row(r, (int)rows, rows_before, lens, slots, a.block_table, a.bt_stride, a.n_pages, p.shift);
        a.out_slot_map[r] = o.at;
        a.out_row_seq[r] = o.seq;
        a.out_row_pos[r] = o.pos;
    }
}

// The rows of a large plan: a CTA takes ROWS of them, finds the slots in shared memory.
constexpr int RW_THREADS = 256, RW_ROWS = 1024;
__global__ void __launch_bounds__(RW_THREADS) plan_rows_kernel(const __grid_constant__ PlanArgs p) {
    extern __shared__ int pg_sm[];  // [slots + 1] rows before each slot, [slots] lengths before the step
    const mtp_page_plan_args& a = p.a;
    const int slots = a.slots, first = blockIdx.x * RW_ROWS;
    int *before = pg_sm, *lens = pg_sm + slots + 1;
    pdl_launch_dependents();
    pdl_wait();
    const int rows = a.out_status[1];
    if (first < rows) {
        for (int s = threadIdx.x; s <= slots; s += RW_THREADS) before[s] = a.out_cu_rows[s];
        __syncthreads();
        for (int s = threadIdx.x; s < slots; s += RW_THREADS) lens[s] = a.out_kv_lens[s] - (before[s + 1] - before[s]);
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < RW_ROWS / RW_THREADS; ++u) {
        const int r = first + u * RW_THREADS + threadIdx.x;
        if (r >= a.max_rows) break;
        const PlanRow o = plan_row(r, rows, before, lens, slots, a.block_table, a.bt_stride, a.n_pages, p.shift);
        a.out_slot_map[r] = o.at;
        a.out_row_seq[r] = o.seq;
        a.out_row_pos[r] = o.pos;
    }
}

// ---- append ----

struct AppendArgs {
    mtp_cache_append_args a;
    int shift;
    unsigned vecs;   // 8-element pieces of a row's keys
    unsigned total;  // rows * 2 * vecs
};

constexpr int AP_THREADS = 256, AP_UNROLL = 4;

template <class DST, int SRC, bool VECTOR>
__device__ __forceinline__ uint4 load8(const void* base, int64_t at) {
    if constexpr (SRC == MTP_F32) {
        const float* p = static_cast<const float*>(base) + at;
        float x[8];
        if constexpr (VECTOR) {
            const float4 u = *reinterpret_cast<const float4*>(p), v = *(reinterpret_cast<const float4*>(p) + 1);
            x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
            x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = *(p + i);
        }
        return make_uint4(DST::pack(x[0], x[1]), DST::pack(x[2], x[3]), DST::pack(x[4], x[5]), DST::pack(x[6], x[7]));
    } else {  // the pool's own type: copied bit by bit
        const uint16_t* p = static_cast<const uint16_t*>(base) + at;
        if constexpr (VECTOR) return *reinterpret_cast<const uint4*>(p);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (uint32_t)*(p + 2 * i) | (uint32_t)*(p + 2 * i + 1) << 16;
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// A thread moves AP_UNROLL pieces of eight elements, all loaded before any is stored.
// Bound by memory: each element is read once and written once.  14592 rows of 16 heads of 64, bf16:
// 120 MB in 17.4 us, 6.9 TB/s (19.3 us a call with other rows between); a step's 128 rows are latency,
// 3.3 us.  VECTOR: rows on 16-byte boundaries are read 16 bytes at a time; the same rows again and
// again 17.5 us a call, element by element 21.5 (from fp32 27.5 and 30.9).
template <class DST, int SRC, bool VECTOR>
__global__ void __launch_bounds__(AP_THREADS) cache_append_kernel(const __grid_constant__ AppendArgs p) {
    const mtp_cache_append_args& a = p.a;
    const unsigned first = blockIdx.x * (AP_THREADS * AP_UNROLL) + threadIdx.x, hv = a.head_dim / 8;
    uint16_t* pool = static_cast<uint16_t*>(a.kv_pool);
    uint4 x[AP_UNROLL];
    uint16_t* to[AP_UNROLL];
    pdl_launch_dependents();
    pdl_wait();
#pragma unroll
    for (int u = 0; u < AP_UNROLL; ++u) {
        const unsigned i = first + u * AP_THREADS;
        to[u] = nullptr;
        if (i >= p.total) continue;
        const unsigned row = i / (2 * p.vecs), rest = i - row * 2 * p.vecs, kv = rest >= p.vecs, vec = rest - kv * p.vecs;
        const int64_t slot = *(a.slot_map + row), page = slot >> p.shift;
        if (slot < 0 || page >= a.n_pages) continue;
        const unsigned head = vec / hv, c = vec - head * hv;
        const int64_t block = ((page * a.layers + a.layer) * 2 + kv) * a.n_kv_heads + head;
        to[u] = pool + ((block << p.shift) + (slot & ((1 << p.shift) - 1))) * a.head_dim + c * 8;
        x[u] = load8<DST, SRC, VECTOR>(kv ? a.v : a.k, (int64_t)row * (kv ? a.v_stride : a.k_stride) + vec * 8);
    }
#pragma unroll
    for (int u = 0; u < AP_UNROLL; ++u)
        if (to[u]) *reinterpret_cast<uint4*>(to[u]) = x[u];
}

template <class DST>
cudaError_t launch_append(const AppendArgs& p, bool vector, cudaStream_t s) {
    const unsigned grid = (p.total + AP_THREADS * AP_UNROLL - 1) / (AP_THREADS * AP_UNROLL);
    const auto kern = p.a.src_dtype == MTP_F32 ? vector ? cache_append_kernel<DST, MTP_F32, true> : cache_append_kernel<DST, MTP_F32, false>
                      : vector                 ? cache_append_kernel<DST, MTP_BF16, true>
                                               : cache_append_kernel<DST, MTP_BF16, false>;
    return launch_ex(kern, dim3(grid), AP_THREADS, 0, s, 1, p);
}

// ---- reorder ----

struct ReorderArgs {
    mtp_beam_reorder_args a;
    int shift;
    int rows;      // batch * beams
    int* count;    // workspace: pages to copy
    int4* copies;  // workspace: {from, to, tokens, -}
};

// One launch of a cluster: checks, new tables, lengths and counts, and the list of copies.
// A page's count is the number of tables that hold it, so the new count is the old one,
// plus the kept beams' holdings, minus the old beams'.  A beam that is its own parent and
// copies nothing adds and takes the same, and is left out.  The additions come first: a
// count passes zero only where no table holds the page any more.
template <int CTAS>
__global__ void __launch_bounds__(PG_THREADS, 1) beam_reorder_kernel(const __grid_constant__ ReorderArgs p) {
    extern __shared__ int pg_sm[];
    __shared__ uint32_t part[PG_WARPS];
    __shared__ int s_free, s_bad, s_freed;
    const mtp_beam_reorder_args& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = CTAS == 1 ? 0 : blockIdx.x, rows = p.rows, W = a.beams;
    int* copies_before = pg_sm;                    // [rows + 1]
    int* from = copies_before + rows + 1;          // [rows]: the parent's row, -1 = none
    int* old = from + rows;                        // [rows]: the length before
    uint32_t* bits = reinterpret_cast<uint32_t*>(old + rows);
    auto lens = [&](int r) { return from[r] < 0 ? 0 : old[from[r]]; };  // the parent's
    const long long cap = (long long)a.bt_stride << p.shift;
    const int part_mask = (1 << p.shift) - 1;

    pdl_launch_dependents();
    pdl_wait();
    uint32_t want = 0;
    bool bad = false;
    if (tid == 0) s_freed = 0;
    for (int r0 = 0; r0 < rows; r0 += PG_THREADS) {
        const int r = r0 + tid;
        uint32_t x = 0, sx;
        if (r < rows) {
            const int item = r / W, j = r - item * W, parent = a.parent[r];
            int n = a.kv_lens[r], src = -1;
            old[r] = n;
            bad |= parent >= W || n < 0 || n > cap;
            n = 0;
            if (parent >= 0 && parent < W) {
                src = item * W + parent;
                n = a.kv_lens[src];
                if (n < 0 || n > cap) n = 0;  // (refused)
                bool again = false;
#pragma unroll 4
                for (int i = 0; i < j; ++i) again |= a.parent[item * W + i] == parent;
                x = again && (n & part_mask);
            }
            from[r] = src;
        }
        x = block_scan(x, part, sx);
        if (r < rows) copies_before[r] = (int)(want + x);
        want += sx;
    }
    if (tid == 0) copies_before[rows] = (int)want;
    bad = __syncthreads_or(bad) != 0;
    // every page that a table holds is one, and is counted (an entry per thread)
    const unsigned stride = a.bt_stride, first = rank * PG_THREADS + tid, step = CTAS * PG_THREADS, entries = rows * stride;
    if (!bad)
#pragma unroll 4
        for (unsigned e = first; e < entries; e += step) {
            const int r = e / stride, c = e - r * stride;
            if (c < pages_of(old[r], p.shift)) {
                const int page = a.block_table[e];
                bad |= page < 0 || page >= a.n_pages || a.page_refs[page] < 1;
            }
        }
    bad = __syncthreads_or(bad) != 0;
    if (tid == 0) s_bad = bad;
    const FreeBits f = find_free<CTAS>(a.page_refs, a.out_page_refs, a.n_pages, rank, bits, part, &s_free);
    team_barrier<CTAS>();  // counts copied, totals there
    long long base;
    const long long free_all = team_sum<CTAS>(&s_free, rank, &base);
    bad = team_sum<CTAS>(&s_bad, rank, nullptr) != 0;
    const int code = bad ? MTP_ERR_INVALID : want > free_all ? MTP_ERR_NO_PAGES : MTP_OK;
    if (code != MTP_OK) {  // everything stays
        for (int r = rank * PG_WARPS + warp; r < rows; r += CTAS * PG_WARPS)
            for (int c = lane; c < a.bt_stride; c += 32)
                a.out_block_table[(size_t)r * a.bt_stride + c] = a.block_table[(size_t)r * a.bt_stride + c];
        for (int r = rank * PG_THREADS + tid; r < rows; r += CTAS * PG_THREADS) a.out_kv_lens[r] = a.kv_lens[r];
        if (rank == 0 && tid == 0) {
            *p.count = 0;
            a.out_status[0] = code;
            a.out_status[1] = 0;
            a.out_status[2] = (int)free_all;
            a.out_status[3] = 0;
        }
        if (CTAS > 1) team_barrier<CTAS>();  // no peer still reads this CTA's shared memory
        return;
    }
    take_free(f, base, want, [&](int page, int n) {
        const int r = owner_of(copies_before, rows + 1, n), tokens = lens(r);
        p.copies[n] = make_int4(a.block_table[(size_t)from[r] * a.bt_stride + (tokens >> p.shift)], page,
                                tokens & part_mask, 0);
        a.out_page_refs[page] = 1;
    });
    team_barrier<CTAS>();  // the copies' pages are known
    auto itself = [&](int r) { return from[r] == r && copies_before[r + 1] == copies_before[r]; };
#pragma unroll 4
    for (unsigned e = first; e < entries; e += step) {
        const int r = e / stride, c = e - r * stride, used = pages_of(lens(r), p.shift);
        int page = -1;
        if (c < used) {
            if (c == used - 1 && copies_before[r + 1] != copies_before[r]) {
                page = __ldcg(&p.copies[copies_before[r]].y);
            } else {
                page = a.block_table[from[r] * stride + c];
                if (!itself(r)) atomicAdd(a.out_page_refs + page, 1);
            }
        }
        a.out_block_table[e] = page;
    }
    team_barrier<CTAS>();
    int freed = 0;
#pragma unroll 4
    for (unsigned e = first; e < entries; e += step) {
        const int r = e / stride, c = e - r * stride;
        if (c < pages_of(old[r], p.shift) && !itself(r))
            freed += atomicSub(a.out_page_refs + a.block_table[e], 1) == 1;
    }
    if (freed) atomicAdd(&s_freed, freed);
    team_barrier<CTAS>();
    for (int r = rank * PG_THREADS + tid; r < rows; r += CTAS * PG_THREADS) a.out_kv_lens[r] = lens(r);
    if (rank == 0 && tid == 0) {
        const long long all = free_all - want + team_sum<CTAS>(&s_freed, rank, nullptr);
        *p.count = (int)want;
        a.out_status[0] = MTP_OK;
        a.out_status[1] = (int)want;
        a.out_status[2] = (int)all;
        a.out_status[3] = 0;
    }
    if (CTAS > 1) team_barrier<CTAS>();  // no peer still reads this CTA's shared memory
}

constexpr int CP_THREADS = 256, CP_UNROLL = 4;

// The filled rows of every copied page: for each (layer, keys | values, head) one run of
// tokens * head_dim elements.  A warp takes a run; CP_UNROLL loads are in flight per lane.
// Bound by memory: each row is read once and written once; with few copies by latency (the list, then
// the rows).  96 beams, 12 layers of 16 heads of 64: 36 copies of 1091 rows, 107 MB read and written,
// 21.2 us a call, of which 15.8 at 6.8 TB/s; 83 and 136 MB 17.4 and 26.0 us, 12.2 and 20.0.  The 5 to 6 us
// above that are the tables', which come before.
__global__ void __launch_bounds__(CP_THREADS) page_copy_kernel(const __grid_constant__ ReorderArgs p, int runs) {
    pdl_launch_dependents();
    pdl_wait();
    const int n = *p.count, lane = threadIdx.x & 31;
    const long long total = (long long)n * runs, stride = (long long)gridDim.x * (CP_THREADS / 32);
    const size_t block = (size_t)p.a.head_dim << p.shift >> 3;  // 16-byte pieces of a (page, layer, K | V, head) block
    uint4* pool = static_cast<uint4*>(p.a.kv_pool);
    for (long long w = (long long)blockIdx.x * (CP_THREADS / 32) + (threadIdx.x >> 5); w < total; w += stride) {
        const int i = (int)(w / runs), run = (int)(w - (long long)i * runs);
        const int4 c = p.copies[i];
        const uint4* src = pool + ((size_t)c.x * runs + run) * block;
        uint4* dst = pool + ((size_t)c.y * runs + run) * block;
        const int pieces = c.z * (p.a.head_dim >> 3);
        for (int q0 = lane; q0 < pieces; q0 += 32 * CP_UNROLL) {
            uint4 v[CP_UNROLL];
#pragma unroll
            for (int u = 0; u < CP_UNROLL; ++u)
                if (q0 + u * 32 < pieces) v[u] = src[q0 + u * 32];
#pragma unroll
            for (int u = 0; u < CP_UNROLL; ++u)
                if (q0 + u * 32 < pieces) dst[q0 + u * 32] = v[u];
        }
    }
}

size_t reorder_workspace(int rows) { return 16 + (size_t)rows * sizeof(int4); }

}  // namespace
}  // namespace mtp

using namespace mtp;

extern "C" {

MTP_API int mtp_page_plan(const mtp_page_plan_args* a, void* cuda_stream) {
    return guarded([&]() -> int {
        if (!a || a->slots < 1 || a->slots > PG_MAX_SLOTS || a->n_pages < 1 || a->n_pages > PG_MAX_PAGES ||
            !page_size_ok(a->page_size) || a->bt_stride < 1 || a->max_rows < 0 || a->max_rows > PG_MAX_ROWS)
            return invalid("page_plan: invalid sizes");
        if ((long long)a->bt_stride * a->page_size > (1 << 30)) return invalid("page_plan: bt_stride %d", a->bt_stride);
        if (!a->kv_lens || !a->new_lens || !a->block_table || !a->page_refs || !a->out_kv_lens || !a->out_page_refs ||
            !a->out_cu_rows || !a->out_status ||
            (a->max_rows > 0 && (!a->out_slot_map || !a->out_row_seq || !a->out_row_pos)))
            return invalid("page_plan: null pointer");
        const bool one = a->n_pages <= PG_ONE_PAGES && a->slots <= PG_ONE_SLOTS && a->max_rows <= PG_ONE_ROWS;
        const PlanArgs p{*a, log2_of(a->page_size), a->max_rows <= PG_ROWS_HERE};
        const size_t smem = (size_t)(3 * a->slots + 2 + 2 * free_words(a->n_pages, one ? 1 : PG_CLUSTER)) * 4;
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        cudaError_t e = one ? launch(page_plan_kernel<1>, 1, PG_THREADS, smem, 1, s, p)
                            : launch(page_plan_kernel<PG_CLUSTER>, PG_CLUSTER, PG_THREADS, smem, PG_CLUSTER, s, p);
        if (e == cudaSuccess && !p.rows_here)
            e = launch(plan_rows_kernel, (a->max_rows + RW_ROWS - 1) / RW_ROWS, RW_THREADS, (size_t)(2 * a->slots + 1) * 4, 1, s, p);
        return cuda_status(e, "page_plan");
    });
}

MTP_API int mtp_cache_append(const mtp_cache_append_args* a, void* cuda_stream) {
    return guarded([&]() -> int {
        if (!a) return invalid("cache_append: null arguments");
        if (const int r = check_pool("cache_append", a->n_pages, a->layers, a->layer, a->n_kv_heads, a->head_dim,
                                     a->page_size))
            return r;
        if (a->rows < 0) return invalid("cache_append: rows %d", a->rows);
        if ((a->pool_dtype != MTP_BF16 && a->pool_dtype != MTP_F16) ||
            (a->src_dtype != MTP_F32 && a->src_dtype != a->pool_dtype))
            return invalid("cache_append: src_dtype %d, pool_dtype %d", a->src_dtype, a->pool_dtype);
        const int width = a->n_kv_heads * a->head_dim;
        if (a->k_stride < width || a->v_stride < width)
            return invalid("cache_append: row strides %lld, %lld below %d", (long long)a->k_stride,
                           (long long)a->v_stride, width);
        const unsigned vecs = width / 8;
        if ((long long)a->rows * 2 * vecs > INT_MAX) return invalid("cache_append: rows %d", a->rows);
        if (a->rows == 0) return MTP_OK;
        if (!a->k || !a->v || !a->slot_map || !a->kv_pool) return invalid("cache_append: null pointer");
        if (!aligned16(a->kv_pool)) return invalid("cache_append: kv_pool must be 16-byte aligned");
        const int size = a->src_dtype == MTP_F32 ? 4 : 2;
        if (reinterpret_cast<uintptr_t>(a->k) % size || reinterpret_cast<uintptr_t>(a->v) % size)
            return invalid("cache_append: k and v must be aligned to their elements");
        AppendArgs p{*a, log2_of(a->page_size), vecs, (unsigned)a->rows * 2 * vecs};
        const bool vector = aligned16(a->k) && aligned16(a->v) && a->k_stride * size % 16 == 0 && a->v_stride * size % 16 == 0;
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        return cuda_status(a->pool_dtype == MTP_BF16 ? launch_append<Bf16>(p, vector, s) : launch_append<F16>(p, vector, s),
                           "cache_append");
    });
}

MTP_API size_t mtp_beam_reorder_workspace_bytes(const mtp_beam_reorder_args* a) {
    if (!a || a->batch < 1 || a->beams < 1 || (long long)a->batch * a->beams > PG_MAX_SLOTS) return 0;
    return reorder_workspace(a->batch * a->beams);
}

MTP_API int mtp_beam_reorder(const mtp_beam_reorder_args* a, void* workspace, size_t workspace_bytes,
                             void* cuda_stream) {
    return guarded([&]() -> int {
        if (!a) return invalid("beam_reorder: null arguments");
        if (const int r = check_pool("beam_reorder", a->n_pages, a->layers, 0, a->n_kv_heads, a->head_dim, a->page_size))
            return r;
        if (a->batch < 1 || a->beams < 1 || a->beams > 64 || (long long)a->batch * a->beams > PG_MAX_SLOTS ||
            a->bt_stride < 1 || (long long)a->bt_stride * a->page_size > (1 << 30) ||
            (long long)a->batch * a->beams * a->bt_stride > (1 << 30))
            return invalid("beam_reorder: invalid sizes (batch %d, beams %d, bt_stride %d)", a->batch, a->beams,
                           a->bt_stride);
        if (a->pool_dtype != MTP_BF16 && a->pool_dtype != MTP_F16)
            return invalid("beam_reorder: pool_dtype %d", a->pool_dtype);
        if (!a->parent || !a->block_table || !a->kv_lens || !a->page_refs || !a->kv_pool || !a->out_block_table ||
            !a->out_kv_lens || !a->out_page_refs || !a->out_status)
            return invalid("beam_reorder: null pointer");
        if (a->out_block_table == a->block_table || a->out_kv_lens == a->kv_lens)
            return invalid("beam_reorder: the new tables and lengths need buffers of their own");
        if (!aligned16(a->kv_pool)) return invalid("beam_reorder: kv_pool must be 16-byte aligned");
        const int rows = a->batch * a->beams;
        if (!workspace || !aligned16(workspace) || workspace_bytes < reorder_workspace(rows))
            return invalid("beam_reorder: workspace %zu bytes, need %zu, 16-byte aligned", workspace_bytes,
                           reorder_workspace(rows));
        const bool one = a->n_pages <= PG_ONE_PAGES && rows <= PG_ONE_BEAMS;
        const ReorderArgs p{*a, log2_of(a->page_size), rows, static_cast<int*>(workspace),
                            reinterpret_cast<int4*>(static_cast<char*>(workspace) + 16)};
        const size_t smem = (size_t)(3 * rows + 1 + 2 * free_words(a->n_pages, one ? 1 : PG_CLUSTER)) * 4;
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        cudaError_t e = one ? launch(beam_reorder_kernel<1>, 1, PG_THREADS, smem, 1, s, p)
                            : launch(beam_reorder_kernel<PG_CLUSTER>, PG_CLUSTER, PG_THREADS, smem, PG_CLUSTER, s, p);
        if (e == cudaSuccess && a->beams > 1) {  // (one beam has nothing to copy)
            int dev = 0, sms = 0;
            e = cudaGetDevice(&dev);
            if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
            if (e == cudaSuccess)
                e = launch(page_copy_kernel, sms * 8, CP_THREADS, 0, 1, s, p, a->layers * 2 * a->n_kv_heads);
        }
        return cuda_status(e, "beam_reorder");
    });
}

}  // extern "C"
