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
#include <climits>
#include <cmath>
#include <type_traits>

#include "serving.cuh"

namespace mtp {
namespace {

constexpr int VF_THREADS = 512, VF_WARPS = VF_THREADS / 32;
constexpr int VF_BLOCK = 256;      // tokens whose weights are summed as one: 8 a lane
template <int TYPE>
constexpr int VF_ITEM = TYPE == MTP_F32 ? 2 : 4;  // blocks that a lane reads at once
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

// The same weights divided by their sum, of 2^-44: l = log2 of it, by its nearest entry of the table and the rest's logarithm.
__device__ __forceinline__ void divide_by(Exponent& e, long long sum, const ExEntry* table) {
    const int zeros = __clzll(sum);
    const unsigned long long m = (unsigned long long)sum << zeros;  // in [1, 2) times 2^63
    const float hi = (float)(uint32_t)(m >> 40) * 0x1p-23f, lo = (float)(uint32_t)(m >> 8) * 0x1p-55f;
    const int k = __float2int_rn(log2f(hi) * EX_STEPS);
    const ExEntry t = table[k & (EX_STEPS - 1)];
    const float two = k >= EX_STEPS ? 2.f : 1.f;
    const float r = ((hi - two * t.hi) + (lo - two * t.lo)) / (two * t.hi);
    e.l_steps = (63 - zeros - 44) * EX_STEPS + k;
    e.l_rest = 1.4426950409f * r * fmaf(-r, fmaf(-r, 0.3333333333f, 0.5f), 1.f);
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
    __device__ __forceinline__ float raw(int token) const { return Logit<TYPE>::get(x + token); }
    __device__ __forceinline__ float at(int token) const { return tame(raw(token)); }
    // places j .. j + 7 (j a multiple of 8) as they stand in memory; -inf outside the row, no token's
    struct Raw {
        uint4 v[TYPE == MTP_F32 ? 2 : 1];
    };
    __device__ __forceinline__ Raw fetch(int j) const {
        Raw r;
        const int first = j - shift;
        if (first >= 0 && first + 8 <= vocab) {
            r.v[0] = *reinterpret_cast<const uint4*>(x + first);
            if constexpr (TYPE == MTP_F32) r.v[1] = *reinterpret_cast<const uint4*>(x + first + 4);
        } else if constexpr (TYPE == MTP_F32) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = in(first + i) ? __float_as_uint(x[first + i]) : 0xff800000u;
            r.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
            r.v[1] = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
            constexpr uint32_t NONE = TYPE == MTP_BF16 ? 0xff80u : 0xfc00u;
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = (in(first + 2 * i) ? (uint32_t)x[first + 2 * i] : NONE) | (in(first + 2 * i + 1) ? (uint32_t)x[first + 2 * i + 1] : NONE) << 16;
            r.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
        }
        return r;
    }
    static __device__ __forceinline__ Raw none() {
        constexpr uint32_t NONE = TYPE == MTP_F32 ? 0xff800000u : TYPE == MTP_BF16 ? 0xff80ff80u : 0xfc00fc00u;
        Raw r;
        r.v[0] = make_uint4(NONE, NONE, NONE, NONE);
        if constexpr (TYPE == MTP_F32) r.v[1] = r.v[0];
        return r;
    }
    static __device__ __forceinline__ void decode(const Raw& r, float (&v)[8]) {
        const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
        if constexpr (TYPE == MTP_F32) {
            const uint32_t y[4] = {r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = __uint_as_float(w[i]);
                v[4 + i] = __uint_as_float(y[i]);
            }
        } else {
            using H = typename std::conditional<TYPE == MTP_BF16, Bf16, F16>::type;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = H::to_float((uint16_t)w[i]);
                v[2 * i + 1] = H::to_float((uint16_t)(w[i] >> 16));
            }
        }
    }
    __device__ __forceinline__ void load(int j, float (&v)[8]) const { decode(fetch(j), v); }
    __device__ __forceinline__ bool in(int token) const { return token >= 0 && token < vocab; }
    // values of places j .. j + 7 that are not finite as those that they count as
    __device__ __forceinline__ void make_tame(int j, float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = in(j - shift + i) ? tame(v[i]) : -INFINITY;
    }
};
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

struct alignas(16) Stat {  // of a row's logits: the largest, sum of 2^((x - top) c), lowest token of the largest
    float top, sum;
    int arg;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Into the shared memory of the cluster's CTA `rank`, at this CTA's place p.
__device__ __forceinline__ void push(long long* p, int rank, long long v) {
    asm volatile("st.shared::cluster.s64 [%0], %1;" ::"r"(dsmem_addr(p, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ void push(Stat* p, int rank, const Stat& s) {
    const uint32_t at = dsmem_addr(p, rank);
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %3};" ::"r"(at), "r"(__float_as_uint(s.top)), "r"(__float_as_uint(s.sum)), "r"(s.arg) : "memory");
}
// Of the lanes' rows one: c as Exponent's.
__device__ __forceinline__ Stat merge(const Stat& s, float c) {
    Stat all;
    all.top = warp_max(s.top);
    all.sum = mtp::warp_sum(s.sum * ex2((s.top - all.top) * c));
    all.arg = __reduce_min_sync(FULL_MASK, s.top == all.top ? s.arg : INT_MAX);
    return all;
}
__device__ __forceinline__ long long warp_scan(long long x) {  // inclusive
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(FULL_MASK, x, o);
        if (lane >= o) x += u;
    }
    return x;
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
        float x[8], y[8];
        const auto raw = t.fetch(j);
        if (mode == DRAW_REST)  // (all on their way together)
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = t.in(j - t.shift + i) ? d.raw(j - t.shift + i) : -INFINITY;
        Row<TYPE>::decode(raw, x);
        t.make_tame(j, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int a, b;
            ex_fixed(x[i], p, table, a, b);
            w[i] = ((long long)a << 22) + b;
            const int token = j - t.shift + i;
            if (mode == DRAW_WITHOUT && token == without) w[i] = 0;
            if (mode == DRAW_REST) {
                ex_fixed(t.in(token) ? tame(y[i]) : -INFINITY, q, table, a, b);
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
    __shared__ Stat parts[2 * VF_MAX_NEW + VF_WARPS], gather[VF_MAX_CLUSTER][2 * VF_MAX_NEW], stat[2 * VF_MAX_NEW];
    __shared__ int state[VF_MAX_NEW];
    __shared__ long long warp_total[2][VF_WARPS], word[2][2][VF_MAX_CLUSTER];
    __shared__ int s_block, s_keep;
    __shared__ long long s_before, s_at;
    const mtp_draft_verify_args& a = p.a;
    ExEntry* table = reinterpret_cast<ExEntry*>(vf_sm);
    long long* block_sum = reinterpret_cast<long long*>(vf_sm + sizeof(ExTable));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, C = p.ctas, slot = blockIdx.x / C, rank = blockIdx.x - slot * C;
    constexpr int ITEM = VF_ITEM<TYPE>;
    const int V = a.vocab;
    pdl_launch_dependents();
    if (C > 1) cluster_arrive_relaxed();  // (before the first push every CTA is there)
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
        if (C > 1) cluster_wait();
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
    // c = log2 e / T as hi + lo.  (All in 32 bits: 64-bit operations of a CTA's threads take microseconds.)
    const float t_tame = fminf(fmaxf(T, 1e-30f), 1e30f), cf = 1.44269502f / t_tame;
    const float c_lo = (fmaf(-cf, t_tame, 1.44269502f) + 1.92596299e-8f) / t_tame;
    const int b0 = rank * p.blocks;  // this CTA's blocks of every row

    // ---- 1: every row's largest logit and sum ----
    const int tasks = n + (drafter ? n - 1 : 0), items = (p.blocks + ITEM - 1) / ITEM, total = tasks * items;
    auto row_of = [&](int task) {
        return task < n ? Row<TYPE>(a.logits, r0 + task, a.logits_stride, V) : Row<TYPE>(a.draft_logits, r0 + task - n, a.draft_stride, V);
    };
    // what the drafts are judged by, on its way
    const int* drafts = a.tokens + r0 + 1;  // [n - 1]
    int draft = -1;
    float draft_u = 0.f, draft_x = 0.f, draft_y = 0.f;
    if (tid < n - 1) {
        draft = drafts[tid];
        draft_u = a.uniforms[2 * (r0 + tid)];
        if (draft >= 0 && draft < V) {
            draft_x = row_of(tid).at(draft);
            if (drafter) draft_y = row_of(n + tid).at(draft);
        }
    }
    auto first_item = [&](int w) { return (int)((long long)total * w / VF_WARPS); };
    for (int it = first_item(warp), stop = first_item(warp + 1); it < stop;) {
        const int task = it / items, from = it, to = min(stop, (task + 1) * items);
        const Row<TYPE> row = row_of(task);
        Stat s;
        // values that are not finite show in the sum or the largest: such a row is gone through once more, with what they count as
#pragma unroll 1
        for (int safe = greedy; safe < 2; ++safe) {
            s = Stat{-VF_HUGE, 0.f, V};
            typename Row<TYPE>::Raw raw[ITEM], next[ITEM];
            auto fetch = [&](int it) {
                const int block = b0 + (it - task * items) * ITEM, stop_block = it < to ? min(b0 + p.blocks, block + ITEM) : 0;
#pragma unroll
                for (int k = 0; k < ITEM; ++k) next[k] = block + k < stop_block ? row.fetch((block + k) * VF_BLOCK + lane * 8) : Row<TYPE>::none();
            };
            fetch(from);
#pragma unroll 1
            for (it = from; it < to; ++it) {
                const int block = b0 + (it - task * items) * ITEM, stop_block = min(b0 + p.blocks, block + ITEM);
                float x[ITEM][8];
                float top = s.top;
#pragma unroll
                for (int k = 0; k < ITEM; ++k) raw[k] = next[k];
                fetch(it + 1);
#pragma unroll
                for (int k = 0; k < ITEM; ++k) Row<TYPE>::decode(raw[k], x[k]);
                if (safe)
#pragma unroll
                    for (int k = 0; k < ITEM; ++k)
                        if (block + k < stop_block) row.make_tame((block + k) * VF_BLOCK + lane * 8, x[k]);
#pragma unroll
                for (int k = 0; k < ITEM; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, x[k][i]);
                if (greedy) {
                    if (top > s.top || s.arg == V) {
                        int arg = V;
#pragma unroll
                        for (int k = ITEM - 1; k >= 0; --k)
#pragma unroll
                            for (int i = 7; i >= 0; --i)
                                if (x[k][i] == top) arg = (block + k) * VF_BLOCK + lane * 8 + i - row.shift;
                        s.arg = arg;
                    }
                } else {
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int k = 0; k < ITEM; ++k)
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            const float2 z = mul2(add2(make_float2(x[k][i], x[k][i + 1]), make_float2(-top, -top)), make_float2(cf, cf));
                            sum[i >> 1 & 1] = add2(sum[i >> 1 & 1], make_float2(ex2(z.x), ex2(z.y)));
                        }
                    s.sum = fmaf(s.sum, ex2((s.top - top) * cf), (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y));
                }
                s.top = top;
            }
            // (a number that no comparison holds for, too)
            if (__all_sync(FULL_MASK, s.sum >= 0.f && s.top < VF_HUGE)) break;
        }
        s = merge(s, cf);
        if (lane == 0) parts[task + warp] = s;
    }
    __syncthreads();
    if (C > 1) cluster_wait();
    for (int task = warp; task < tasks; task += VF_WARPS) {  // a lane per warp's part, then per CTA
        const bool has = lane < VF_WARPS && max(first_item(lane), task * items) < min(first_item(lane + 1), (task + 1) * items);
        const Stat s = merge(has ? parts[task + lane] : Stat{-VF_HUGE, 0.f, V}, cf);
        if (lane < C) push(&gather[rank][task], lane, s);
    }
    team();
    for (int task = warp; task < tasks; task += VF_WARPS) {
        Stat s = merge(lane < C ? gather[lane][task] : Stat{-VF_HUGE, 0.f, V}, cf);
        if (!(s.top > -VF_HUGE)) s.sum = (float)V;  // nothing above what -infinity counts as: all alike
        if (lane == 0) stat[task] = s;
    }
    __syncthreads();

    // ---- 2: the drafts ----
    if (tid < n - 1) {
        int keep = 0;
        if (draft >= 0 && draft < V) {
            if (greedy) {
                keep = stat[tid].arg == draft;
            } else {
                const float q = drafter ? ex2((draft_y - stat[n + tid].top) * cf) : 1.f, q_sum = drafter ? stat[n + tid].sum : 1.f;
                const float l = unit(draft_u) * q * stat[tid].sum, r = ex2((draft_x - stat[tid].top) * cf) * q_sum;
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
        e.c_lo = c_lo;
        e.l_steps = 0;
        e.l_rest = 0.f;
        return e;
    };
    int turn = 0;  // which of the words the next sum over the CTAs uses
    // sums over the cluster of the warps' totals, and the first one's over the CTAs before this one
    auto all_sums = [&](long long (&all)[2], long long& before) {
        __syncthreads();
        if (warp < 2) {
            long long t = lane < VF_WARPS ? warp_total[warp][lane] : 0;
#pragma unroll
            for (int o = VF_WARPS / 2; o > 0; o >>= 1) t += __shfl_xor_sync(FULL_MASK, t, o);
            if (lane < C) push(&word[turn][warp][rank], lane, t);
        }
        team();
        all[0] = all[1] = before = 0;
#pragma unroll
        for (int r = 0; r < VF_MAX_CLUSTER; ++r) {
            if (r >= C) break;
            const long long t = word[turn][0][r];
            if (r < rank) before += t;
            all[0] += t;
            all[1] += word[turn][1][r];
        }
        turn ^= 1;
    };
    int kept = 0;
    bool cut = false;
    long long sums[2] = {0, 0}, before;  // of the weights of the row after the kept ones, the target's and the drafter's, in 2^-44
    while (kept < n - 1) {
        int keep = state[kept];
        if (keep == 2 || (keep == 0 && drafter)) {
            // the blocks of both rows, one after another; the next one's on their way
            const Row<TYPE> rows[2] = {row_of(kept), row_of(drafter ? n + kept : kept)};
            const Exponent zs[2] = {exponent(kept), exponent(drafter ? n + kept : kept)};
            const int count = p.blocks * (1 + drafter);
            auto fetch = [&](int k) {
                const int e = k >= p.blocks;
                return k < count ? (e ? rows[1] : rows[0]).fetch((b0 + k - e * p.blocks) * VF_BLOCK + lane * 8) : Row<TYPE>::none();
            };
            typename Row<TYPE>::Raw next = fetch(warp);
            long long sum[2] = {0, 0};
#pragma unroll 1
            for (int k = warp; k < count; k += VF_WARPS) {
                const bool e = k >= p.blocks;
                const Row<TYPE> row = e ? rows[1] : rows[0];
                const Exponent z = e ? zs[1] : zs[0];
                float x[8];
                Row<TYPE>::decode(next, x);
                next = fetch(k + VF_WARPS);
                row.make_tame((b0 + k - e * p.blocks) * VF_BLOCK + lane * 8, x);
                int sa = 0, sb = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    int u, v;
                    ex_fixed(x[i], z, table, u, v);
                    sa += u;
                    sb += v;
                }
                const long long s = ((long long)sa << 22) + sb;
                sum[0] += e ? 0 : s;
                sum[1] += e ? s : 0;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum[e] += __shfl_xor_sync(FULL_MASK, sum[e], o);
                if (lane == 0) warp_total[e][warp] = sum[e];
            }
            all_sums(sums, before);
        }
        if (keep == 2) {
            if (tid == 0) {
                const int d = drafts[kept];
                auto probability = [&](int task, long long sum) {
                    const double z = ((double)row_of(task).at(d) - (double)stat[task].top) * (1.4426950408889634 / (double)t_tame);
                    return exp2(z) / ((double)sum * 0x1p-44);
                };
                s_keep = (double)unit(a.uniforms[2 * (r0 + kept)]) * (drafter ? probability(n + kept, sums[1]) : 1.0) < probability(kept, sums[0]);
            }
            __syncthreads();
            keep = s_keep;
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
        if (draw.mode == DRAW_REST) {  // by the sums: both distributions in the same units
            draw.q = exponent(n + kept);
            divide_by(draw.p, sums[0], table);
            divide_by(draw.q, sums[1], table);
        }
        const Row<TYPE> t = row_of(kept), d = draw.mode == DRAW_REST ? row_of(n + kept) : t;
        if (tid == 0) s_block = -1;
        const float number = unit(a.uniforms[2 * (r0 + kept) + 1]);
        // 0: sums of all blocks; 1: where there are none, those of the target alone; 2: the block that the number falls into
        long long at = 0;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            long long total = 0;
#pragma unroll 1
            for (int k = pass < 2 ? warp : warp == 0 ? s_block : -1; k >= 0 && k < p.blocks; k += VF_WARPS) {
                long long w[8], s = 0;
                const int j = (b0 + k) * VF_BLOCK + lane * 8;
                draw.weights(t, d, table, j, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) s += w[i];
                if (pass < 2) {
                    // (s < 2^48: two parts whose sums over a warp have 32 bits)
                    const uint32_t lo = __reduce_add_sync(FULL_MASK, (uint32_t)s & ((1u << 26) - 1)), hi = __reduce_add_sync(FULL_MASK, (uint32_t)(s >> 26));
                    s = ((long long)hi << 26) + lo;
                    if (lane == 0) block_sum[k] = s;
                    total += s;
                    continue;
                }
                long long x = warp_scan(s) + s_before - s;
                int found = V;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x += w[i];
                    if (x > at && found == V) found = j - t.shift + i;
                }
                token = __reduce_min_sync(FULL_MASK, found);
                break;
            }
            if (pass == 2) break;
            __syncthreads();  // (earlier sums are still read)
            if (lane == 0) {
                warp_total[0][warp] = total;
                warp_total[1][warp] = 0;
            }
            long long all[2];
            all_sums(all, before);
            if (all[0] == 0 && pass == 0) {  // nothing is left of p: p
                draw.mode = DRAW_TARGET;
                draw.p.l_steps = 0;
                draw.p.l_rest = 0.f;
                continue;
            }
            // the token's weight covers this place
            if (tid == 0) s_at = min((long long)((double)number * (double)all[0]), all[0] - 1) - before;
            __syncthreads();
            at = s_at;
            if (warp == 0 && at >= 0) {
                long long base = 0;
                for (int k0 = 0; k0 < p.blocks; k0 += 32) {
                    const int k = k0 + lane;
                    const long long s = k < p.blocks ? block_sum[k] : 0, x = base + warp_scan(s);
                    if (x > at && x - s <= at) {
                        s_block = k;
                        s_before = x - s;
                    }
                    base = __shfl_sync(FULL_MASK, x, 31);
                }
                __syncwarp();
            }
            pass = 1;
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
        while (ctas < VF_MAX_CLUSTER && (long long)a->slots * ctas * 2 <= 2 * sms && a->vocab / (ctas * 2) >= VF_BLOCK * 4) ctas *= 2;
        const int most = 16 / size - 1;  // places before a row's first token
        const int blocks = (a->vocab + most + VF_BLOCK - 1) / VF_BLOCK;
        const DraftArgs p{*a, a->block_table ? log2_of(a->page_size) : 0, ctas, (blocks + ctas - 1) / ctas};
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        e = a->logits_dtype == MTP_F32 ? launch_verify<MTP_F32>(p, s) : a->logits_dtype == MTP_BF16 ? launch_verify<MTP_BF16>(p, s) : launch_verify<MTP_F16>(p, s);
        return cuda_status(e, "draft_verify");
    });
}

}  // extern "C"
