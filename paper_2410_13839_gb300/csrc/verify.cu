// verify.cu -- which drafted tokens the target's distribution keeps, the token after them, and
// the pages of what is not kept (mtp_draft_verify).
//
//   p = softmax(x / T), q = softmax(y / T) of the drafter (or all on the drafted token);
//   draft d of a row is kept where u q(d) < p(d); after the first that is not, token t is drawn from
//   max(p - q, 0), after the last one kept from p: the first t with sum_{i <= t} w_i > v sum_i w_i.
//
// A cluster of CTAs has a slot: each takes a part of the vocabulary of every row, the parts meet over
// distributed shared memory, and no workspace is needed.
//   1  maxima and sums of exponentials of all rows, in fp32, one pass (memory bounds it);
//   2  the drafts are judged by every CTA alike.  fp32 leaves out the comparisons closer than
//      1e-4: those rows' sums are made again as in 3;
//   3  the drawn row's weights, as sums of blocks of 256 tokens, then the block that v falls into,
//      then the token.
// Between the 48001 borders of such a draw lie 2e-5 of it each, and a sum in fp32 may be off by more
// than a hundredth of that, so step 3's weights are whole numbers of 2^-44 (with T = 1024 parts of a power of two
// in a table and a polynomial for the rest, 2^z to about 2^-36): their sums are exact and the same in any order, so
// the outcome depends on nothing but the inputs.  (fp64 exponentials would do the same at a fiftieth of the rate.)
#include <algorithm>
#include <cmath>

#include "serving.cuh"

namespace mtp {
namespace {

constexpr int VF_THREADS = 512, VF_WARPS = VF_THREADS / 32;
constexpr int VF_BLOCK = 256;      // tokens whose weights are summed as one: 8 a lane
constexpr int VF_ITEM = 4;         // blocks that a lane has in flight
constexpr int VF_MAX_NEW = 64, VF_MAX_VOCAB = 1 << 18, VF_MAX_CLUSTER = 8;
constexpr float VF_HUGE = 1e38f;   // infinite logits count as this
constexpr float VF_NEAR = 1e-4f;   // products nearer than this, relatively, are compared in 64 bits

// ---- 2^z as a whole number of 2^-44 ----

constexpr int EX_BITS = 10, EX_STEPS = 1 << EX_BITS;  // 2^(j / 1024) = hi + lo
struct alignas(8) ExEntry {
    float hi, lo;
};
struct ExTable {
    ExEntry e[EX_STEPS];
};
constexpr ExTable make_ex_table() {
    ExTable t{};
    for (int j = 0; j < EX_STEPS; ++j) {
        const double x = j * 0.69314718055994530942 / EX_STEPS;
        double term = 1.0, sum = 1.0;
        for (int n = 1; n < 24; ++n) {
            term *= x / n;
            sum += term;
        }
        t.e[j].hi = (float)sum;
        t.e[j].lo = (float)(sum - (double)t.e[j].hi);
    }
    return t;
}
__device__ const ExTable ex_table = make_ex_table();

// A distribution's exponents: z = (x - top) c - l, c = log2 e / T as hi + lo, l = steps / 1024 + l_rest.
struct Exponent {
    float top;
    float c_hi, c_lo;
    int l_steps;
    float l_rest;
};
// 2^z = a 2^-22 + b 2^-44, a <= 2^22, |b| <= 2^21 + 1: two roundings to fixed steps by adding a constant of the step's size.
__device__ __forceinline__ void ex_fixed(float x, const Exponent& e, const ExEntry* table, int& a, int& b) {
    // x - top as d + err, exactly
    const float d = x - e.top, bb = d - x, err = (x - (d - bb)) + (-e.top - bb);
    const float p = d * e.c_hi;
    float rest = fmaf(d, e.c_hi, -p);
    rest = fmaf(d, e.c_lo, rest);
    rest = fmaf(err, e.c_hi, rest);
    constexpr float ROUND = 12582912.f;  // 1.5 * 2^23
    const float kf = fmaf(p, (float)EX_STEPS, ROUND);
    const int k = __float_as_int(kf) - __float_as_int(ROUND) - e.l_steps;
    const float r = fmaf(kf - ROUND, -1.f / EX_STEPS, p) + (rest - e.l_rest);
    const ExEntry t = table[k & (EX_STEPS - 1)];
    const float scale = __int_as_float((max(k >> EX_BITS, -126) + 127) << 23);
    // 2^r - 1, |r| < 2^-10: ln 2 r + (ln 2 r)^2 / 2 + (ln 2 r)^3 / 6
    const float m = r * fmaf(r, fmaf(r, 0.0555041087f, 0.2402265070f), 0.6931471806f);
    const float hi = t.hi * scale, lo = fmaf(t.hi, m, t.lo) * scale;
    const float u = (hi + lo) + 3.f;  // steps of 2^-22 above 2
    const float left = (hi - (u - 3.f)) + lo;
    const float v = fmaf(left, 0x1p44f, ROUND);
    const bool there = p > -100.f;  // (below nothing is left; -inf gives no number)
    a = there ? __float_as_int(u) - __float_as_int(3.f) : 0;
    b = there ? __float_as_int(v) - __float_as_int(ROUND) : 0;
}

// ---- rows ----

struct DraftArgs {
    mtp_draft_verify_args a;
    int shift;   // page_size = 1 << shift
    int ctas;    // CTAs of a slot
    int blocks;  // blocks of a CTA's part of a row
};

template <int TYPE>
struct Logit;
template <>
struct Logit<MTP_F32> {
    using type = float;
    static __device__ __forceinline__ float get(const float* p) { return *p; }
};
template <>
struct Logit<MTP_BF16> {
    using type = uint16_t;
    static __device__ __forceinline__ float get(const uint16_t* p) { return Bf16::to_float(*p); }
};
template <>
struct Logit<MTP_F16> {
    using type = uint16_t;
    static __device__ __forceinline__ float get(const uint16_t* p) { return F16::to_float(*p); }
};
__device__ __forceinline__ float unit(float u) { return u > 0.f ? fminf(u, 1.f) : 0.f; }  // NaN: 0
__device__ __forceinline__ float tame(float x) { return fminf(fmaxf(x, -VF_HUGE), VF_HUGE); }  // NaN: the lowest

// A row of logits.  Its blocks begin at the 16-byte boundary at or before the row: place j is token j - shift.
template <int TYPE>
struct Row {
    const typename Logit<TYPE>::type* x;
    int shift, vocab;
    __device__ __forceinline__ Row(const void* base, long long row, long long stride, int n) : vocab(n) {
        x = static_cast<const typename Logit<TYPE>::type*>(base) + row * stride;
        shift = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(*x));
    }
    __device__ __forceinline__ float at(int token) const { return tame(Logit<TYPE>::get(x + token)); }
    // places j .. j + 7 (j a multiple of 8); -inf outside the row: no token's
    __device__ __forceinline__ void load(int j, float (&v)[8]) const {
        const int first = j - shift;
        if (first >= 0 && first + 8 <= vocab) {
            if constexpr (TYPE == MTP_F32) {
                const float4 p = *reinterpret_cast<const float4*>(x + first), q = *reinterpret_cast<const float4*>(x + first + 4);
                v[0] = p.x; v[1] = p.y; v[2] = p.z; v[3] = p.w;
                v[4] = q.x; v[5] = q.y; v[6] = q.z; v[7] = q.w;
            } else {
                using H = typename std::conditional<TYPE == MTP_BF16, Bf16, F16>::type;
                const uint4 p = *reinterpret_cast<const uint4*>(x + first);
                const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[2 * i] = H::to_float((uint16_t)w[i]);
                    v[2 * i + 1] = H::to_float((uint16_t)(w[i] >> 16));
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = tame(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = first + i >= 0 && first + i < vocab ? at(first + i) : -INFINITY;
        }
    }
};

struct Stat {  // of a row's logits: the largest, sum of 2^((x - top) c), lowest token of the largest
    float top, sum;
    int arg;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ long long ld_cluster_i64(const long long* p, int rank) {
    long long v;
    asm volatile("ld.shared::cluster.s64 %0, [%1];" : "=l"(v) : "r"(dsmem_addr(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ float ld_cluster_f32(const float* p, int rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(dsmem_addr(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ int ld_cluster_i32(const int* p, int rank) {
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(dsmem_addr(p, rank)) : "memory");
    return v;
}

// How the weights of a draw are made.
enum DrawMode { DRAW_TARGET, DRAW_WITHOUT, DRAW_REST };  // p; p but for the drafted token; max(p - q, 0)

template <int TYPE>
struct Draw {
    DrawMode mode;
    int without;
    Exponent p, q;
    // weights of places j .. j + 7 of the target's row
    __device__ __forceinline__ void weights(const Row<TYPE>& t, const Row<TYPE>& d, const ExEntry* table, int j, long long (&w)[8]) const {
        float x[8];
        t.load(j, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int a, b;
            ex_fixed(x[i], p, table, a, b);
            w[i] = ((long long)a << 22) + b;
            const int token = j - t.shift + i;
            if (mode == DRAW_WITHOUT && token == without) w[i] = 0;
            if (mode == DRAW_REST) {
                const bool in = token >= 0 && token < t.vocab;
                ex_fixed(in ? d.at(token) : -INFINITY, q, table, a, b);
                w[i] -= ((long long)a << 22) + b;
            }
            w[i] = w[i] > 0 ? w[i] : 0;
        }
    }
};

// Grid (slots * ctas).  Shared memory: the table, [2 max_new] sums of rows and of their segments, sums of blocks.
template <int TYPE>
__global__ void __launch_bounds__(VF_THREADS, 2) draft_verify_kernel(const __grid_constant__ DraftArgs p) {
    extern __shared__ __align__(16) unsigned char vf_sm[];
    __shared__ Stat parts[2 * VF_MAX_NEW + VF_WARPS], mine[2 * VF_MAX_NEW], stat[2 * VF_MAX_NEW];
    __shared__ int state[VF_MAX_NEW];
    __shared__ long long warp_total[VF_WARPS], word[2];
    __shared__ int s_block, s_keep;
    __shared__ long long s_before;
    const mtp_draft_verify_args& a = p.a;
    ExEntry* table = reinterpret_cast<ExEntry*>(vf_sm);
    long long* block_sum = reinterpret_cast<long long*>(vf_sm + sizeof(ExTable));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, C = p.ctas, slot = blockIdx.x / C, rank = blockIdx.x - slot * C;
    const int V = a.vocab;
    pdl_launch_dependents();
    for (int i = tid; i < EX_STEPS; i += VF_THREADS) table[i] = ex_table.e[i];
    pdl_wait();
    auto team = [&]() {
        if (C > 1) {
            cluster_arrive_release();
            cluster_wait();
        } else {
            __syncthreads();
        }
    };
    const int r0 = a.cu_rows[slot], end = a.cu_rows[slot + 1], n = end - r0, len = a.kv_lens[slot];
    const bool bad = r0 < 0 || n < 0 || end > a.rows || n > a.max_new || len < n ||
                     (a.block_table && len > (long long)a.bt_stride << p.shift);
    int* out = a.out_tokens + (long long)slot * a.max_new;
    if (bad || n == 0) {  // (the whole cluster)
        if (rank == 0) {
            for (int i = tid; i < a.max_new; i += VF_THREADS) out[i] = -1;
            if (tid == 0) {
                a.out_counts[slot] = 0;
                a.out_kv_lens[slot] = len;
                if (a.out_done) a.out_done[slot] = 0;
                if (bad && a.err_word) atomicOr(a.err_word, ERR_BOUNDS);
            }
        }
        return;
    }
    const float T = a.temperature ? a.temperature[slot] : 1.f;
    const bool greedy = !(T > 0.f), drafter = a.draft_logits && !greedy;
    const double c = 1.4426950408889634 / fmin(fmax((double)T, 1e-30), 1e30);
    const float cf = (float)c;
    const int b0 = rank * p.blocks;  // this CTA's blocks of every row

    // ---- 1: every row's largest logit and sum ----
    const int tasks = n + (drafter ? n - 1 : 0), items = (p.blocks + VF_ITEM - 1) / VF_ITEM, total = tasks * items;
    auto row_of = [&](int task) {
        return task < n ? Row<TYPE>(a.logits, r0 + task, a.logits_stride, V) : Row<TYPE>(a.draft_logits, r0 + task - n, a.draft_stride, V);
    };
    auto first_item = [&](int w) { return (int)((long long)total * w / VF_WARPS); };
    for (int it = first_item(warp), stop = first_item(warp + 1); it < stop;) {
        const int task = it / items, to = min(stop, (task + 1) * items);
        const Row<TYPE> row = row_of(task);
        Stat s{-VF_HUGE, 0.f, V};
        for (; it < to; ++it) {
            const int block = b0 + (it - task * items) * VF_ITEM, stop_block = min(b0 + p.blocks, block + VF_ITEM);
            float x[VF_ITEM][8];
            float top = s.top;
#pragma unroll
            for (int k = 0; k < VF_ITEM; ++k) {
                if (block + k < stop_block) {
                    row.load((block + k) * VF_BLOCK + lane * 8, x[k]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[k][i] = -INFINITY;
                }
            }
#pragma unroll
            for (int k = 0; k < VF_ITEM; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, x[k][i]);
            if (greedy) {
                if (top > s.top || s.arg == V) {
                    int arg = V;
#pragma unroll
                    for (int k = VF_ITEM - 1; k >= 0; --k)
#pragma unroll
                        for (int i = 7; i >= 0; --i) {
                            const int token = (block + k) * VF_BLOCK + lane * 8 + i - row.shift;
                            if (x[k][i] == top && block + k < stop_block && token >= 0 && token < V) arg = token;
                        }
                    s.arg = arg;
                }
            } else {
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int k = 0; k < VF_ITEM; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[i & 1] += ex2((x[k][i] - top) * cf);
                s.sum = fmaf(s.sum, ex2((s.top - top) * cf), sum[0] + sum[1]);
            }
            s.top = top;
        }
        const float top = warp_max(s.top);
        const float sum = mtp::warp_sum(s.sum * ex2((s.top - top) * cf));
        const int arg = __reduce_min_sync(FULL_MASK, s.top == top ? s.arg : V);
        if (lane == 0) parts[task + warp] = Stat{top, sum, arg};
    }
    __syncthreads();
    if (tid < tasks) {
        Stat s{-VF_HUGE, 0.f, V};
        for (int w = 0; w < VF_WARPS; ++w) {
            if (max(first_item(w), tid * items) >= min(first_item(w + 1), (tid + 1) * items)) continue;
            const Stat x = parts[tid + w];
            const float top = fmaxf(s.top, x.top);
            s.sum = s.sum * ex2((s.top - top) * cf) + x.sum * ex2((x.top - top) * cf);
            s.arg = min(s.top == top ? s.arg : V, x.top == top ? x.arg : V);
            s.top = top;
        }
        mine[tid] = s;
    }
    team();
    if (tid < tasks) {
        Stat s{-VF_HUGE, 0.f, V};
        for (int r = 0; r < C; ++r) {
            const Stat x{ld_cluster_f32(&mine[tid].top, r), ld_cluster_f32(&mine[tid].sum, r), ld_cluster_i32(&mine[tid].arg, r)};
            const float top = fmaxf(s.top, x.top);
            s.sum = s.sum * ex2((s.top - top) * cf) + x.sum * ex2((x.top - top) * cf);
            s.arg = min(s.top == top ? s.arg : V, x.top == top ? x.arg : V);
            s.top = top;
        }
        stat[tid] = s;
    }
    __syncthreads();

    // ---- 2: the drafts ----
    const int* drafts = a.tokens + r0 + 1;  // [n - 1]
    if (tid < n - 1) {
        const int d = drafts[tid];
        int keep = 0;
        if (d >= 0 && d < V) {
            if (greedy) {
                keep = stat[tid].arg == d;
            } else {
                const float u = unit(a.uniforms[2 * (r0 + tid)]);
                float q = 1.f, q_sum = 1.f;
                if (drafter) {
                    q = ex2((row_of(n + tid).at(d) - stat[n + tid].top) * cf);
                    q_sum = stat[n + tid].sum;
                }
                const float l = u * q * stat[tid].sum, r = ex2((row_of(tid).at(d) - stat[tid].top) * cf) * q_sum;
                keep = l < r;
                const float big = fmaxf(l, r);
                if (!(fabsf(l - r) > VF_NEAR * big) || big < 1e-25f) keep = 2;  // too near for 32 bits
            }
        }
        state[tid] = keep;
    }
    __syncthreads();

    auto exponent = [&](int task) {
        Exponent e;
        e.top = stat[task].top;
        e.c_hi = cf;
        e.c_lo = (float)(c - (double)cf);
        e.l_steps = 0;
        e.l_rest = 0.f;
        return e;
    };
    int turn = 0;  // whose word the next sum over the CTAs uses
    // the sum over the cluster of this CTA's total (in warp_total), and of those before it
    auto all_sum = [&](long long& before) {
        __syncthreads();
        if (tid == 0) {
            long long t = 0;
            for (int w = 0; w < VF_WARPS; ++w) t += warp_total[w];
            word[turn] = t;
        }
        team();
        long long all = 0;
        before = 0;
        for (int r = 0; r < C; ++r) {
            const long long t = ld_cluster_i64(&word[turn], r);
            if (r < rank) before += t;
            all += t;
        }
        turn ^= 1;
        return all;
    };
    // the sum of a row's weights, in 2^-44
    auto exact_sum = [&](int task) {
        const Row<TYPE> row = row_of(task);
        const Exponent e = exponent(task);
        long long sum = 0;
        for (int k = warp; k < p.blocks; k += VF_WARPS) {
            float x[8];
            row.load((b0 + k) * VF_BLOCK + lane * 8, x);
            int sa = 0, sb = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                int u, v;
                ex_fixed(x[i], e, table, u, v);
                sa += u;
                sb += v;
            }
            sum += ((long long)sa << 22) + sb;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(FULL_MASK, sum, o);
        __syncthreads();  // (an earlier sum is still read)
        if (lane == 0) warp_total[warp] = sum;
        long long before;
        return all_sum(before);
    };
    auto probability = [&](int task, int token, long long sum) {  // in 64 bits
        return exp2(((double)row_of(task).at(token) - (double)stat[task].top) * c) / ((double)sum * 0x1p-44);
    };

    int kept = 0;
    bool cut = false;
    while (kept < n - 1) {
        int keep = state[kept];
        if (keep == 2) {
            const int d = drafts[kept];
            const long long sp = exact_sum(kept), sq = drafter ? exact_sum(n + kept) : 0;
            if (tid == 0) {
                const double q = drafter ? probability(n + kept, d, sq) : 1.0;
                s_keep = (double)unit(a.uniforms[2 * (r0 + kept)]) * q < probability(kept, d, sp);
            }
            __syncthreads();
            keep = s_keep;
            __syncthreads();
        }
        if (!keep) break;
        ++kept;
        if (drafts[kept - 1] == a.eos_id) {
            cut = true;
            break;
        }
    }

    // ---- 3: the token ----
    int token = V;  // V: not this CTA's
    if (!cut && greedy) {
        token = rank == 0 ? stat[kept].arg : V;
    } else if (!cut) {
        Draw<TYPE> draw;
        const bool refused = kept < n - 1;
        draw.mode = !refused ? DRAW_TARGET : drafter ? DRAW_REST : DRAW_WITHOUT;
        draw.without = refused ? drafts[kept] : -1;
        draw.p = draw.q = exponent(kept);
        if (draw.mode == DRAW_REST) {
            draw.q = exponent(n + kept);
            auto divide = [](Exponent& e, long long sum) {  // by the sum: both distributions in the same units
                const double l = log2((double)sum) - 44.0, steps = rint(l * EX_STEPS);
                e.l_steps = (int)steps;
                e.l_rest = (float)(l - steps / EX_STEPS);
            };
            const long long sp = exact_sum(kept), sq = exact_sum(n + kept);
            divide(draw.p, sp);
            divide(draw.q, sq);
        }
        const Row<TYPE> t = row_of(kept), d = draw.mode == DRAW_REST ? row_of(n + kept) : t;
        long long before, all, sum;
        for (;;) {
            sum = 0;
            for (int k = warp; k < p.blocks; k += VF_WARPS) {
                long long w[8], s = 0;
                draw.weights(t, d, table, (b0 + k) * VF_BLOCK + lane * 8, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) s += w[i];
                // (s < 2^48: two parts whose sums over a warp have 32 bits)
                const uint32_t lo = __reduce_add_sync(FULL_MASK, (uint32_t)s & ((1u << 26) - 1)), hi = __reduce_add_sync(FULL_MASK, (uint32_t)(s >> 26));
                s = ((long long)hi << 26) + lo;
                if (lane == 0) block_sum[k] = s;
                sum += s;
            }
            __syncthreads();  // (an earlier sum is still read)
            if (lane == 0) warp_total[warp] = sum;
            all = all_sum(before);
            if (all > 0 || draw.mode == DRAW_TARGET) break;
            draw.mode = DRAW_TARGET;  // nothing is left of p: p
            draw.p.l_steps = 0;
            draw.p.l_rest = 0.f;
        }
        const float v = unit(a.uniforms[2 * (r0 + kept) + 1]);
        const long long at = min((long long)((double)v * (double)all), all - 1) - before;  // the token's weight covers this place
        if (tid == 0) s_block = -1;
        __syncthreads();
        if (warp == 0 && at >= 0) {
            long long base = 0;
            for (int k0 = 0; k0 < p.blocks; k0 += 32) {
                const int k = k0 + lane;
                const long long s = k < p.blocks ? block_sum[k] : 0;
                long long x = s;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const long long u = __shfl_up_sync(FULL_MASK, x, o);
                    if (lane >= o) x += u;
                }
                if (base + x > at && base + x - s <= at) {
                    s_block = k;
                    s_before = base + x - s;
                }
                base += __shfl_sync(FULL_MASK, x, 31);
            }
            __syncwarp();
            const int k = s_block;
            if (k >= 0) {
                long long w[8], s = 0;
                const int j = (b0 + k) * VF_BLOCK + lane * 8;
                draw.weights(t, d, table, j, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) s += w[i];
                long long x = s;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const long long u = __shfl_up_sync(FULL_MASK, x, o);
                    if (lane >= o) x += u;
                }
                x += s_before - s;
                int found = V;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x += w[i];
                    if (x > at && found == V) found = j - t.shift + i;
                }
                token = __reduce_min_sync(FULL_MASK, found);
            }
        }
    }
    if (tid == 0 && token < V) {  // one thread of the cluster
        out[kept] = token;
        if (a.out_done) a.out_done[slot] = token == a.eos_id;
    }

    // ---- the other outputs; the pages of what is not kept ----
    if (rank == C - 1) {
        const int after = len - (n - 1 - kept);
        for (int i = tid; i < a.max_new; i += VF_THREADS)
            if (i != kept || cut) out[i] = i < kept ? drafts[i] : -1;
        if (tid == 0) {
            a.out_counts[slot] = cut ? kept : kept + 1;
            a.out_kv_lens[slot] = after;
            if (cut && a.out_done) a.out_done[slot] = 1;
        }
        if (a.block_table) {
            const int mask = (1 << p.shift) - 1, from = (after + mask) >> p.shift, to = (len + mask) >> p.shift;
            for (int i = from + tid; i < to; i += VF_THREADS) {
                int* entry = a.block_table + (long long)slot * a.bt_stride + i;
                const int page = *entry;
                if (page < 0) continue;
                *entry = -1;
                if (page < a.n_pages && atomicSub(a.page_refs + page, 1) >= 1) continue;
                if (page < a.n_pages) atomicAdd(a.page_refs + page, 1);  // it was free already
                if (a.err_word) atomicOr(a.err_word, ERR_BOUNDS);
            }
        }
    }
    if (C > 1) team();  // no peer still reads this CTA's shared memory
}

template <int TYPE>
cudaError_t launch_verify(const DraftArgs& p, cudaStream_t s) {
    const size_t smem = sizeof(ExTable) + (size_t)p.blocks * sizeof(long long);
    return launch(draft_verify_kernel<TYPE>, p.a.slots * p.ctas, VF_THREADS, smem, p.ctas, s, p);
}

}  // namespace
}  // namespace mtp

using namespace mtp;

extern "C" {

MTP_API int mtp_draft_verify(const mtp_draft_verify_args* a, void* cuda_stream) {
    return guarded([&]() -> int {
        if (!a || a->slots < 1 || a->slots > 8192 || a->rows < 0 || a->vocab < 1 || a->vocab > VF_MAX_VOCAB || a->max_new < 1 ||
            a->max_new > VF_MAX_NEW)
            return invalid("draft_verify: invalid sizes (slots, rows, vocab or max_new)");
        if (a->logits_dtype != MTP_F32 && a->logits_dtype != MTP_BF16 && a->logits_dtype != MTP_F16)
            return invalid("draft_verify: logits_dtype %d", a->logits_dtype);
        if (a->eos_id < -1 || a->eos_id >= a->vocab) return invalid("draft_verify: eos_id %d of %d", a->eos_id, a->vocab);
        if (a->logits_stride < a->vocab || (a->draft_logits && a->draft_stride < a->vocab))
            return invalid("draft_verify: row strides %lld, %lld below %d", (long long)a->logits_stride, (long long)a->draft_stride,
                           a->vocab);
        if (!a->cu_rows || !a->kv_lens || !a->out_tokens || !a->out_counts || !a->out_kv_lens ||
            (a->rows > 0 && (!a->logits || !a->tokens || !a->uniforms)))
            return invalid("draft_verify: null pointer");
        if (!a->block_table != !a->page_refs) return invalid("draft_verify: block_table and page_refs go together");
        if (a->block_table && (!page_size_ok(a->page_size) || a->n_pages < 1 || a->n_pages > PG_MAX_PAGES || a->bt_stride < 1 ||
                               (long long)a->bt_stride * a->page_size > (1 << 30)))
            return invalid("draft_verify: invalid cache (page_size %d, pages %d, bt_stride %d)", a->page_size, a->n_pages, a->bt_stride);
        const int size = a->logits_dtype == MTP_F32 ? 4 : 2;
        if (reinterpret_cast<uintptr_t>(a->logits) % size || reinterpret_cast<uintptr_t>(a->draft_logits) % size ||
            reinterpret_cast<uintptr_t>(a->uniforms) % 4)
            return invalid("draft_verify: logits, draft_logits and uniforms must be aligned to their elements");
        int dev = 0, sms = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) {
            cudaGetLastError();
            return cuda_status(e, "draft_verify");
        }
        // CTAs of a slot: as long as two of them have room on an SM, and their parts of a row are a few blocks
        int ctas = 1;
        while (ctas < VF_MAX_CLUSTER && (long long)a->slots * ctas * 2 <= 2 * sms && a->vocab / (ctas * 2) >= VF_BLOCK * VF_ITEM) ctas *= 2;
        const int most = 16 / size - 1;  // places before a row's first token
        const int blocks = (a->vocab + most + VF_BLOCK - 1) / VF_BLOCK;
        const DraftArgs p{*a, a->block_table ? log2_of(a->page_size) : 0, ctas, (blocks + ctas - 1) / ctas};
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        e = a->logits_dtype == MTP_F32 ? launch_verify<MTP_F32>(p, s) : a->logits_dtype == MTP_BF16 ? launch_verify<MTP_BF16>(p, s) : launch_verify<MTP_F16>(p, s);
        return cuda_status(e, "draft_verify");
    });
}

}  // extern "C"
