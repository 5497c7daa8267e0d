// beam.cu -- beam search's selection (mtp_beam_select): of an item's beams * vocab
// continuations the k best,
//   score(b, t) = beam_score[b] + (logit[b][t] - lse[b]),
// each operation one fp32 operation, by descending score and, where scores are equal,
// ascending b * vocab + t.  A finished beam has one continuation, its end, at its own
// score.
//
// A continuation is a 64-bit key, the score's bits in an order-preserving form above the
// complement of its number: keys are distinct, so the k largest are one set, whatever
// order they are looked at in, and no tie is a special case.
//
// The best keys of a CTA (best_of): a thread goes through its own keys once for their maximum (of 16
// bytes of logits the largest score, then its place);
// 128 groups of threads give a maximum each; the k-th largest of these is a bound that at least
// k keys reach, and hardly more do (for k = 8 about 8.3 are expected, for k = 64 about 89).  The
// few threads with a key that reaches it go through theirs again, and what they find is ranked
// by counting.  Where more than CAND_MAX keys reach it (runs of equal scores that one group
// holds), the keys are taken out one by one instead.
//
// The logits of a long item are not stored anywhere: the second look is L2's.  (Kept in shared
// memory as scores, 32 x 4 beams of 48001 took 21 us: the stores of 16-byte pieces conflict.)  An item
// is cut into segments that make one wave of CTAs; each leaves its k best keys in the workspace,
// and the item's CTA that finishes last (an atomic counter, reset by it) selects among these.
// Short items are one segment; where their log-sum-exp is not given they are held in shared
// memory, and it is taken in the same launch.  Longer items have a kernel for it before, whose
// reading leaves the logits in L2.
//
// What bounds it is latency: a dozen steps with a barrier between them, and for a cut item the way
// of the keys through the workspace.  1 x 5 beams of 1025 fp32 logits, log-sum-exp included: 6.2 us
// a call; 32 x 4 beams of 48001 bf16 logits with theirs given: 13.9 us (12 MB, 1.8 us at 6.8 TB/s).
#include <float.h>

#include <algorithm>

#include "serving.cuh"

namespace mtp {
namespace {

constexpr int BS_THREADS = 512, BS_WARPS = BS_THREADS / 32;
// Most scores of an item held in shared memory.  Held, and with a launch of its own for the log-sum-exp, us a call: 5 beams of
// 1025 6.2 and 8.9, 8 of 1500 8.7 and 10.8.
constexpr int HELD = 14336;
// Scores of an item that is not cut.  Whole and cut: 5125 scores 6.1 and 7.4, 10,000 6.1 and 6.7, 12,000 8.4 and 7.3,
// 40,000 12.2 and 8.3.
constexpr int WHOLE = 10240;
// Fewest scores of a segment (1 x 4 beams of 48001, segments of 1024, 2048, 4096 at least: 11.5, 9.5, 11.1 us); CTAs of a wave
// per SM (32 x 4 beams of 48001, 1 to 4: 20.8, 14.1, 17.4, 20.3 us).
constexpr int LEAST = 2048, SEL_PER_SM = 2;
constexpr int GROUPS = 128;       // groups of four threads, each with a maximum
constexpr int CAND_MAX = 1024, HELD_KEYS = 1024;
constexpr int BS_MAX_K = 64, BS_MAX_BEAMS = 64, BS_MAX_BATCH = 4096;
constexpr int LSE_THREADS = 512;

struct SelectArgsB {
    mtp_beam_select_args a;
    int segments, seg_len;        // segments of an item, scores of a segment
    const float* lse;             // given, or a kernel's before this one
    unsigned long long* keys;     // [batch][segments][k]
    int* count;                   // [batch]
};

// A score as it is ranked: NaN is -inf, -0 is 0.
__device__ __forceinline__ float ranked(float score) { return isnan(score) ? -INFINITY : score + 0.f; }
__device__ __forceinline__ unsigned long long make_key(float score, uint32_t number) {
    uint32_t u = __float_as_uint(score);
    u ^= (u >> 31) ? 0xffffffffu : 0x80000000u;
    return (unsigned long long)u << 32 | (0xffffffffu - number);
}
__device__ __forceinline__ float key_score(unsigned long long key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ unsigned long long warp_max64(unsigned long long v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(FULL_MASK, v, o));
    return v;
}

struct Best {
    unsigned long long thread_max[BS_THREADS];
    unsigned long long group_max[GROUPS];
    unsigned long long cand[CAND_MAX];
    unsigned long long best[BS_MAX_K];
    unsigned long long held[HELD_KEYS];  // the segments' keys, when they are joined
    unsigned long long bound, warp_best[BS_WARPS];
    int n;
};

// The k largest of the block's keys into b.best, descending; 0 past the last.  each(f) calls f with
// every key of this thread; `most`: their largest (0: none).  The whole block calls it; b.best is
// visible afterwards.
template <class EACH>
__device__ __forceinline__ void best_of(Best& b, int k, unsigned long long most, EACH each) {
    static_assert(BS_THREADS == 4 * GROUPS, "four threads to a group");
    const int tid = threadIdx.x;
    b.thread_max[tid] = most;
    if (tid == 0) {
        b.bound = 1;  // fewer than k groups with a key: all keys
        b.n = 0;
    }
    if (tid < BS_MAX_K) b.best[tid] = 0;
    __syncthreads();
    // (threads far apart: a short segment's keys are with the first warps)
    if (tid < GROUPS)
        b.group_max[tid] = max(max(b.thread_max[tid], b.thread_max[tid + GROUPS]),
                               max(b.thread_max[tid + 2 * GROUPS], b.thread_max[tid + 3 * GROUPS]));
    __syncthreads();
    const unsigned long long mine = b.group_max[tid >> 2];
    int larger = 0;  // a quarter of the groups to a thread
#pragma unroll
    for (int i = tid & 3; i < GROUPS; i += 4) larger += b.group_max[i] > mine;
    larger += __shfl_xor_sync(FULL_MASK, larger, 1);
    larger += __shfl_xor_sync(FULL_MASK, larger, 2);
    if ((tid & 3) == 0 && larger == k - 1 && mine) b.bound = mine;
    __syncthreads();
    const unsigned long long bound = b.bound;
    if (most >= bound)
        each([&](unsigned long long x) {
            if (x >= bound) {
                const int at = atomicAdd(&b.n, 1);
                if (at < CAND_MAX) b.cand[at] = x;
            }
        });
    __syncthreads();
    const int found = b.n;
    if (found <= CAND_MAX) {
        for (int i = tid; i < found; i += BS_THREADS) {
            const unsigned long long x = b.cand[i];
            int larger = 0;
#pragma unroll 4
            for (int j = 0; j < found; ++j) larger += b.cand[j] > x;
            if (larger < k) b.best[larger] = x;
        }
        __syncthreads();
        return;
    }
    unsigned long long last = ~0ull;
    for (int r = 0; r < k && last; ++r) {
        unsigned long long x = 0;
        each([&](unsigned long long y) {
            if (y < last) x = max(x, y);
        });
        __syncwarp();
        x = warp_max64(x);
        if ((tid & 31) == 0) b.warp_best[tid >> 5] = x;
        __syncthreads();
        x = 0;
#pragma unroll
        for (int w = 0; w < BS_WARPS; ++w) x = max(x, b.warp_best[w]);
        if (tid == 0) b.best[r] = x;
        last = x;
        __syncthreads();
    }
}

struct F32T {
    using elem = float;
    static constexpr int PER = 4;
    static __device__ __forceinline__ float one(const void* p, int64_t i) { return *(static_cast<const float*>(p) + i); }
    static __device__ __forceinline__ void unpack(uint4 v, float* x) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
};
template <class T>
struct Half {
    using elem = uint16_t;
    static constexpr int PER = 8;
    static __device__ __forceinline__ float one(const void* p, int64_t i) {
        return T::to_float(*(static_cast<const uint16_t*>(p) + i));
    }
    static __device__ __forceinline__ void unpack(uint4 v, float* x) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = T::to_float((uint16_t)w[i]);
            x[2 * i + 1] = T::to_float((uint16_t)(w[i] >> 16));
        }
    }
};

// piece(i, x) for the elements [0, n) at p + first, x[0 .. T::PER - 1] those from i on, by `warps` warps of which this
// is number `warp`: 16 bytes at a time, UNROLL loads in flight, each warp a stretch of 32 UNROLL pieces; the
// single elements before the first and after the last 16-byte boundary, one(i, x), by warp 0.  Returns the stretches there are.
template <class T, int UNROLL, class F, class G>
__device__ __forceinline__ int for_pieces(const void* base, int64_t first, int n, int warp, int warps, F one, G piece) {
    using E = typename T::elem;
    const E* p = static_cast<const E*>(base) + first;
    const int lane = threadIdx.x & 31;
    const int head = min(n, (int)(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(E)));
    const int vecs = (n - head) / T::PER, rest = head + vecs * T::PER + lane;
    if (warp == 0 && lane < head) one(lane, T::one(p, lane));
    const uint4* v = reinterpret_cast<const uint4*>(p + head);
    for (int i0 = warp * (32 * UNROLL) + lane; i0 - lane < vecs; i0 += warps * (32 * UNROLL)) {
        uint4 raw[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
            if (i0 + u * 32 < vecs) raw[u] = *(v + i0 + u * 32);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int i = i0 + u * 32;
            if (i < vecs) {
                float x[T::PER];
                T::unpack(raw[u], x);
                piece(head + i * T::PER, x);
            }
        }
    }
    if (warp == 0 && rest < n) one(rest, T::one(p, rest));
    return max(1, (vecs + 32 * UNROLL - 1) / (32 * UNROLL));
}

// (maximum, sum of exp(x - maximum)) of two sets, as one.  The maximum passes NaN over, the sum keeps it.
__device__ __forceinline__ void join_sums(float& m, float& s, float m2, float s2) {
    const float top = fmaxf(m, m2);
    if (top == -INFINITY) {  // neither has a value: each sum is 0, or NaN
        s += s2;
        return;
    }
    s = s * __expf(m - top) + s2 * __expf(m2 - top);
    m = top;
}

// log-sum-exp of a row, a cluster of CTAs each (one where the rows fill the GPU): a running maximum and sum per thread, moved
// once per 16 bytes, so that their exponentials do not wait for each other.  Bound by latency: a selection from 128
// rows of 48001 bf16 logits takes 22.3 us with it, 13.9 where the log-sum-exps are given (37.5 with a step per
// element).  Clusters of 8 and one CTA per row: 24 rows of 48001 18.5 and 21.0 us, one row 11.8 and 12.9; of 2 and one: 24
// rows of 5000 15.8 and 14.9.
constexpr int LSE_CLUSTER = 8, LSE_LEAST = 4096;  // most CTAs of a row; fewest elements of a part
template <class T>
__global__ void __launch_bounds__(LSE_THREADS) row_lse_kernel(const void* logits, int64_t stride, int vocab, int ctas,
                                                              float* out) {
    __shared__ float2 part[LSE_THREADS / 32];
    __shared__ float s_max, s_sum;
    const int row = blockIdx.x / ctas, rank = blockIdx.x - row * ctas, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int seg = ((vocab + ctas - 1) / ctas + 7) & ~7, first = min(vocab, rank * seg), n = min(seg, vocab - first);
    pdl_launch_dependents();
    pdl_wait();
    float m = -INFINITY, s = 0.f;
    auto raise = [&](float top) {
        if (top > m) {
            s *= __expf(m - top);  // (the first value: 0)
            m = top;
        }
        return m == -INFINITY ? 0.f : m;
    };
    for_pieces<T, 4>(
        logits, row * stride + first, n, warp, LSE_THREADS / 32,
        [&](int, float x) {
            const float ref = raise(x);
            s += __expf(x - ref);
        },
        [&](int, const float (&x)[T::PER]) {
            float top = x[0], sum = 0.f;
#pragma unroll
            for (int e = 1; e < T::PER; ++e) top = fmaxf(top, x[e]);
            const float ref = raise(top);
#pragma unroll
            for (int e = 0; e < T::PER; ++e) sum += __expf(x[e] - ref);
            s += sum;
        });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        join_sums(m, s, __shfl_xor_sync(FULL_MASK, m, o), __shfl_xor_sync(FULL_MASK, s, o));
    if (lane == 0) part[warp] = make_float2(m, s);
    __syncthreads();
    if (warp == 0) {
        const float2 q = lane < LSE_THREADS / 32 ? part[lane] : make_float2(-INFINITY, 0.f);
        m = q.x;
        s = q.y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            join_sums(m, s, __shfl_xor_sync(FULL_MASK, m, o), __shfl_xor_sync(FULL_MASK, s, o));
        if (lane == 0) {
            s_max = m;
            s_sum = s;
        }
    }
    if (ctas > 1) {
        __syncthreads();
        cluster_arrive_release();
        cluster_wait();
        if (rank == 0 && warp == 0) {
            m = lane < ctas ? ld_dsmem(dsmem_addr(&s_max, lane)) : -INFINITY;
            s = lane < ctas ? ld_dsmem(dsmem_addr(&s_sum, lane)) : 0.f;
#pragma unroll
            for (int o = LSE_CLUSTER / 2; o > 0; o >>= 1)
                join_sums(m, s, __shfl_xor_sync(FULL_MASK, m, o), __shfl_xor_sync(FULL_MASK, s, o));
        }
    }
    if (rank == 0 && threadIdx.x == 0) out[row] = s != s ? NAN : m + logf(s);  // (nothing but -inf: -inf)
    if (ctas > 1) {  // no peer still reads this CTA's shared memory
        __syncwarp();
        cluster_arrive_release();
        cluster_wait();
    }
}

template <class T, bool HOLD>
__global__ void __launch_bounds__(BS_THREADS) beam_select_kernel(const __grid_constant__ SelectArgsB p) {
    extern __shared__ float bs_score[];  // HOLD: the item's scores
    __shared__ Best b;
    __shared__ float s_lse[BS_MAX_BEAMS], s_beam[BS_MAX_BEAMS];
    __shared__ int s_done[BS_MAX_BEAMS], s_last;
    const mtp_beam_select_args& a = p.a;
    const int item = blockIdx.y, seg = blockIdx.x, W = a.beams, V = a.vocab, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int first = seg * p.seg_len, n = min(p.seg_len, W * V - first);
    pdl_launch_dependents();
    pdl_wait();
    // (held logits are on their way while the beams' scores are)
    float beam_score = 0.f, beam_lse = 0.f;
    int beam_done = 0;
    if (tid < W) {
        beam_score = a.scores[item * W + tid];
        beam_done = a.done ? a.done[item * W + tid] : 0;
        if (!HOLD) beam_lse = p.lse[item * W + tid];
    }
    auto beams_there = [&]() {
        if (tid < W) {
            s_beam[tid] = beam_score;
            s_done[tid] = beam_done;
            if (!HOLD) s_lse[tid] = beam_lse;
        }
        __syncthreads();
    };
    if constexpr (!HOLD) beams_there();
    // one(beam, column, logit) or piece(beam, column, logits) for this thread's logits of the segment, by ascending number; the
    // beams' stretches go round the warps, so that short rows are on their way together.  A finished beam has its end alone.
    auto logits = [&](auto one, auto piece) {
        const int beam0 = first / V, beam1 = (first + n - 1) / V;
        int turn = warp;
        for (int w = beam0; w <= beam1; ++w) {
            const int c0 = max(0, first - w * V), c1 = min(V, first + n - w * V);
            if (s_done[w] && !HOLD) {
                for (int c = c0 + tid; c < c1; c += BS_THREADS) one(w, c, c == a.eos_id ? 0.f : -INFINITY);
            } else {
                const int used = for_pieces<T, 4>(
                    a.logits, ((int64_t)item * W + w) * a.logits_stride + c0, c1 - c0, turn, BS_WARPS,
                    [&](int i, float x) { one(w, c0 + i, x); }, [&](int i, const float (&x)[T::PER]) { piece(w, c0 + i, x); });
                turn = (turn + BS_WARPS - used % BS_WARPS) % BS_WARPS;
            }
        }
    };
    auto each_logit = [&](auto use) {
        logits(use, [&](int w, int c, const float (&x)[T::PER]) {
#pragma unroll
            for (int e = 0; e < T::PER; ++e) use(w, c + e, x[e]);
        });
    };
    if constexpr (HOLD) {  // a warp per beam: its log-sum-exp, then its scores
        each_logit([&](int w, int c, float x) { bs_score[w * V + c] = x; });
        beams_there();
        for (int w = warp; w < W; w += BS_WARPS) {
            float* x = bs_score + w * V;
            float m = -INFINITY, s = 0.f;
#pragma unroll 8
            for (int i = lane; i < V; i += 32) m = fmaxf(m, x[i]);
            m = warp_max(m);
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll 8
            for (int i = lane; i < V; i += 32) s += __expf(x[i] - ref);
            s = warp_sum(s);
            const float lse = m + logf(s), cum = s_beam[w];
            if (lane == 0) s_lse[w] = lse;
            const bool done = s_done[w];
#pragma unroll 8
            for (int i = lane; i < V; i += 32) x[i] = ranked(!done ? cum + (x[i] - lse) : i == a.eos_id ? cum : -INFINITY);
        }
        __syncthreads();
    }
    if (seg == 0 && a.out_lse && tid < W) a.out_lse[item * W + tid] = s_lse[tid];
    // this thread's largest score, the first of equal ones
    float most = -INFINITY;
    uint32_t at_most = 0xffffffffu;
    auto larger = [&](uint32_t number, float x) {  // (numbers ascend)
        if (x > most || at_most == 0xffffffffu) {
            most = x;
            at_most = number;
        }
    };
    int beam = -1;  // (a finished beam's end comes as 0, its score is the beam's own)
    float cum = 0.f, lse = 0.f;
    auto score = [&](int w, float x) {
        if (w != beam) {
            beam = w;
            cum = s_beam[w];
            lse = s_done[w] ? 0.f : s_lse[w];
        }
        return cum + (x - lse);
    };
    auto each = [&](auto f) {  // f(number, score)
        if constexpr (HOLD) {
#pragma unroll 8
            for (int i = tid; i < n; i += BS_THREADS) f((uint32_t)i, bs_score[i]);
        } else {
            each_logit([&](int w, int c, float x) { f((uint32_t)(w * V + c), ranked(score(w, x))); });
        }
    };
    if constexpr (HOLD) {
        each(larger);
    } else {
        logits([&](int w, int c, float x) { larger((uint32_t)(w * V + c), ranked(score(w, x))); },
               [&](int w, int c, const float (&x)[T::PER]) {  // the largest of a piece, then its place
                   float y[T::PER], top = -INFINITY;
#pragma unroll
                   for (int e = 0; e < T::PER; ++e) {
                       y[e] = score(w, x[e]);
                       top = fmaxf(top, y[e]);
                   }
                   if (top > most || at_most == 0xffffffffu) {
                       most = ranked(top);
                       int at = 0;
#pragma unroll
                       for (int e = T::PER - 1; e >= 0; --e) at = ranked(y[e]) == most ? e : at;
                       at_most = (uint32_t)(w * V + c + at);
                   }
               });
    }
    __syncwarp();
    best_of(b, a.k, at_most != 0xffffffffu ? make_key(most, at_most) : 0ull,
            [&](auto f) { each([&](uint32_t number, float x) { f(make_key(x, number)); }); });

    if (p.segments > 1) {
        unsigned long long* keys = p.keys + (size_t)item * p.segments * a.k;
        if (tid < a.k) __stcg(keys + (size_t)seg * a.k + tid, b.best[tid]);
        __threadfence();
        __syncthreads();
        if (tid == 0) s_last = atomicAdd(p.count + item, 1) == p.segments - 1;
        __syncthreads();
        if (!s_last) return;
        __threadfence();
        if (tid == 0) p.count[item] = 0;
        // the k best of all segments' keys, as many at a time as shared memory holds beside the best so far
        unsigned long long* held = b.held;
        const int room = HELD_KEYS, total = p.segments * a.k;
        int have = 0;
        for (int at = 0; at < total;) {
            const int take = min(room - have, total - at);
            for (int i = tid; i < take; i += BS_THREADS) held[have + i] = __ldcg(keys + at + i);
            __syncthreads();
            if (total <= BS_THREADS) {  // few: each finds its rank among all
                if (tid < BS_MAX_K) b.best[tid] = 0;
                __syncthreads();
                if (tid < total && held[tid]) {
                    const unsigned long long x = held[tid];
                    int larger = 0;
#pragma unroll 8
                    for (int j = 0; j < total; ++j) larger += held[j] > x;
                    if (larger < a.k) b.best[larger] = x;
                }
                __syncthreads();
                break;
            }
            unsigned long long most = 0;
            for (int i = tid; i < have + take; i += BS_THREADS) most = max(most, held[i]);
            best_of(b, a.k, most, [&](auto f) {
                for (int i = tid; i < have + take; i += BS_THREADS) f(held[i]);
            });
            at += take;
            have = a.k;
            if (at < total) {
                if (tid < a.k) held[tid] = b.best[tid];
                __syncthreads();
            }
        }
    }
    if (tid < a.k) {
        const unsigned long long key = b.best[tid];
        const uint32_t number = 0xffffffffu - (uint32_t)key;
        const int parent = (int)(number / (uint32_t)V), token = (int)(number - (uint32_t)parent * V);
        const size_t at = (size_t)item * a.k + tid;
        a.out_scores[at] = key_score(key);
        a.out_parent[at] = parent;
        a.out_token[at] = token;
        if (a.out_done) a.out_done[at] = token == a.eos_id || s_done[parent];
    }
}

struct SelectPlan {
    int segments, seg_len, sms;
    bool lse_here, lse_before;
    size_t count_bytes, key_bytes, need;
};

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

int select_plan(const mtp_beam_select_args* a, SelectPlan* p) {
    if (!a || a->batch < 1 || a->batch > BS_MAX_BATCH || a->beams < 1 || a->beams > BS_MAX_BEAMS || a->vocab < 1 ||
        (long long)a->beams * a->vocab > (1 << 30) || a->k < 1 || a->k > BS_MAX_K ||
        (long long)a->k > (long long)a->beams * a->vocab)
        return invalid("beam_select: invalid sizes");
    if (a->logits_dtype != MTP_F32 && a->logits_dtype != MTP_BF16 && a->logits_dtype != MTP_F16)
        return invalid("beam_select: logits_dtype %d", a->logits_dtype);
    const int all = a->beams * a->vocab;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        sms = 152;  // (the sizes are checked all the same; a launch will say what is wrong)
    }
    p->sms = sms;
    // as many segments as make one wave, none shorter than LEAST; short items are one
    p->lse_here = !a->lse && all <= HELD;
    p->segments = p->lse_here || all <= WHOLE ? 1 : std::max(1, std::min((all + LEAST - 1) / LEAST, SEL_PER_SM * sms / a->batch));
    p->seg_len = ((all + p->segments - 1) / p->segments + 7) & ~7;  // even segments
    p->segments = (all + p->seg_len - 1) / p->seg_len;
    p->lse_before = !a->lse && !p->lse_here;
    // the counters' place is the same for all calls, and they are left zero
    p->count_bytes = p->segments > 1 || p->lse_before ? BS_MAX_BATCH * sizeof(int) : 0;
    p->key_bytes = p->segments > 1 ? align256((size_t)a->batch * p->segments * a->k * 8) : 0;
    p->need = p->count_bytes + p->key_bytes +
              (p->lse_before && !a->out_lse ? align256((size_t)a->batch * a->beams * sizeof(float)) : 0);
    return MTP_OK;
}

template <class T>
cudaError_t launch_select(const mtp_beam_select_args* a, const SelectPlan& pl, char* ws, cudaStream_t s) {
    SelectArgsB p{*a, pl.segments, pl.seg_len, a->lse, reinterpret_cast<unsigned long long*>(ws + pl.count_bytes),
                  reinterpret_cast<int*>(ws)};
    if (pl.lse_before) {
        const int rows = a->batch * a->beams;
        float* lse = a->out_lse ? a->out_lse : reinterpret_cast<float*>(ws + pl.count_bytes + pl.key_bytes);
        p.lse = lse;
        p.a.out_lse = nullptr;  // written already
        // clusters while they make no more than two CTAs per SM, none with a part below LSE_LEAST
        int ctas = 1;
        while (ctas < LSE_CLUSTER && rows * ctas * 2 <= pl.sms * 2 && a->vocab / (ctas * 2) >= LSE_LEAST) ctas *= 2;
        const cudaError_t e = launch_ex(row_lse_kernel<T>, dim3(rows * ctas), LSE_THREADS, 0, s, ctas, a->logits,
                                        a->logits_stride, (int)a->vocab, ctas, lse);
        if (e != cudaSuccess) return e;
    }
    const size_t smem = pl.lse_here ? (size_t)pl.seg_len * sizeof(float) : 0;
    const auto kern = pl.lse_here ? beam_select_kernel<T, true> : beam_select_kernel<T, false>;
    const cudaError_t e = pl.lse_here ? ensure_kernel_smem(reinterpret_cast<const void*>(kern), smem) : cudaSuccess;
    if (e != cudaSuccess) return e;
    return launch_ex(kern, dim3(pl.segments, a->batch), BS_THREADS, smem, s, 1, p);
}

}  // namespace
}  // namespace mtp

using namespace mtp;

extern "C" {

MTP_API size_t mtp_beam_select_workspace_bytes(const mtp_beam_select_args* a) {
    SelectPlan p;
    size_t need = 0;
    guarded([&]() -> int {
        const int r = select_plan(a, &p);
        need = r == MTP_OK ? p.need : 0;
        return r;
    });
    return need;
}

MTP_API int mtp_beam_select(const mtp_beam_select_args* a, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return guarded([&]() -> int {
        SelectPlan p;
        if (const int r = select_plan(a, &p)) return r;
        if (!a->logits || !a->scores || !a->out_scores || !a->out_parent || !a->out_token)
            return invalid("beam_select: null pointer");
        if (a->logits_stride < a->vocab) return invalid("beam_select: logits_stride %lld below the vocabulary", (long long)a->logits_stride);
        if (a->eos_id >= a->vocab) return invalid("beam_select: eos_id %d", a->eos_id);
        if (a->done && a->eos_id < 0) return invalid("beam_select: finished beams need an eos_id");
        if (reinterpret_cast<uintptr_t>(a->logits) % (a->logits_dtype == MTP_F32 ? 4 : 2))
            return invalid("beam_select: logits must be aligned to their elements");
        if (p.need && (!workspace || !aligned16(workspace) || workspace_bytes < p.need))
            return invalid("beam_select: workspace %zu bytes, need %zu, 16-byte aligned", workspace_bytes, p.need);
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        char* ws = static_cast<char*>(workspace);
        const cudaError_t e = a->logits_dtype == MTP_F32    ? launch_select<F32T>(a, p, ws, s)
                              : a->logits_dtype == MTP_BF16 ? launch_select<Half<Bf16>>(a, p, ws, s)
                                                            : launch_select<Half<F16>>(a, p, ws, s);
        return cuda_status(e, "beam_select");
    });
}

}  // extern "C"
