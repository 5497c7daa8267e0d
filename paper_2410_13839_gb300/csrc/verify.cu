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
//      1e-4 (and what large exponents add to that): those rows' sums are made again as in 3;
//   3  the drawn row's weights, as sums of blocks of 256 tokens, then the block that v falls into,
//      then the token.
// Between the 48001 borders of such a draw lie 2e-5 of it each, and a sum in fp32 may be off by more
// than a hundredth of that, so step 3's weights are whole numbers of 2^-44 (with 1024 parts of a power of two
// in a table and a polynomial for the rest, 2^z to about 2^-36): their sums are exact and the same in any order, so
// the outcome depends on nothing but the inputs.  They are made once and kept in shared memory, 45 bits each; the weights of
// max(p - q, 0) are p's times q's sum less q's times p's sum, without a division; where they add up to no more than what the
// weights' own errors leave of two that are the same, there is nothing to draw from but p.  (64-bit operations, two a cycle
// and SM, took 15 us of a call where every thread made a logarithm.)
//
// Latency bounds it: three exchanges over the cluster, one after another, of about a microsecond each, and between them a
// chain of 40 operations a weight, 8 to a thread at once.  32 slots of up to 9 rows, 48001 tokens, bf16 (29 MB): 30 us, as
// long as its slot of 9 rows (of 36 us, in an earlier form, phase 1 took 11 to 14, the weights of both rows 13, the draw 6).
// One slot, 5 rows of 32003: 14, of 128256 21; 32 slots, 4 rows of 1025: 8.1.  Where a CTA's part of a row has more blocks than
// shared memory holds the weights of, they are made again in every pass: 32 slots, 4 rows of 48001 24, of 50257 47, of 128256 75.
// Code that is not in the instruction cache costs more than it saves: unrolled and inlined it was 128 KB.
#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>

#include "serving.cuh"

namespace mtp {
namespace {

constexpr int VF_BLOCK = 256;      // tokens that are summed as one: 8 a lane
template <int TYPE>
constexpr int VF_ITEM = TYPE == MTP_F32 ? 2 : 4;  // blocks that a lane reads at once
template <int NT>
constexpr int VF_WINDOW = NT / 32 * 3;  // blocks whose weights shared memory holds: 73 KB and 148 KB
constexpr int VF_MAX_NEW = 64, VF_MAX_VOCAB = 1 << 18, VF_MAX_CLUSTER = 16;
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

// A distribution's exponents: z = x c - l, c = log2 e / T as hi + lo, l = top c as steps / 1024 + rest.
struct Exponent {
    float c_hi, c_lo;
    float low;      // of x: below it nothing of 2^-44 is left
    int steps;      // with the bits of the constant that rounds to whole steps
    float rest;
    float top;      // where products with c are too large for that: subtracted from x first, exactly
    bool wide;
};
constexpr float EX_ROUND = 12582912.f;  // 1.5 * 2^23
__device__ __forceinline__ Exponent make_exponent(float top, float c_hi, float c_lo) {
    Exponent e;
    e.c_hi = c_hi;
    e.c_lo = c_lo;
    e.top = top;
    const float p = top * c_hi;
    e.wide = !(fabsf(p) < 2000.f);  // (2^21 steps; what infinite logits count as passes it at every temperature)
    e.low = (e.wide ? 0.f : top) - 100.f / c_hi;
    const float kf = fmaf(p, (float)EX_STEPS, EX_ROUND);
    e.steps = __float_as_int(EX_ROUND);
    e.rest = 0.f;
    if (!e.wide) {
        e.steps = __float_as_int(kf);
        e.rest = fmaf(kf - EX_ROUND, -1.f / EX_STEPS, p) + fmaf(top, c_lo, fmaf(top, c_hi, -p));
    }
    return e;
}
__device__ __forceinline__ float tame(float x) { return fminf(fmaxf(x, -VF_HUGE), VF_HUGE); }  // NaN: the lowest
// 2^z = (u - 3) + v 2^-44, u in steps of 2^-22, v of 1 with EX_ROUND in front: two roundings to fixed steps by adding a
// constant of the step's size.  Weights add up in the bits of u and v, each a constant too large.
constexpr int EX_U = 0x40400000, EX_V = 0x4b400000;  // bits of 3 and EX_ROUND
__device__ __noinline__ float2 ex_widen(float x, float top, float low, float c) {
    x = tame(x);
    const float d = x - top, bb = d - x;  // x - top = d + err
    return make_float2(d, d > low ? ((x - (d - bb)) + (-top - bb)) * c : 0.f);
}
// table: its address in shared memory.
__device__ __forceinline__ void ex_fixed(float x, const Exponent& e, uint32_t table, int& u_bits, int& v_bits) {
    float err = 0.f;
    if (e.wide) {
        const float2 y = ex_widen(x, e.top, e.low, e.c_hi);
        x = y.x;
        err = y.y;
    }
    x = fmaxf(x, e.low);  // (-inf and NaN, too)
    const float p = x * e.c_hi;
    const float kf = fmaf(p, (float)EX_STEPS, EX_ROUND);
    const int k = __float_as_int(kf) - e.steps;
    const float r = fmaf(kf - EX_ROUND, -1.f / EX_STEPS, p) + ((fmaf(x, e.c_lo, -e.rest) + err) + fmaf(x, e.c_hi, -p));
    ExEntry t;
    asm("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(t.hi), "=f"(t.lo) : "r"(table + (k & (EX_STEPS - 1)) * 8));
    const float scale = __int_as_float((int)((unsigned)k << (23 - EX_BITS) & 0xff800000u) + (127 << 23));
    // 2^r - 1, |r| < 2^-9: ln 2 r + (ln 2 r)^2 / 2 + (ln 2 r)^3 / 6
    const float m = r * fmaf(r, fmaf(r, 0.0555041087f, 0.2402265070f), 0.6931471806f);
    const float hi = t.hi * scale, lo = fmaf(t.hi, m, t.lo) * scale;
    const float u = (hi + lo) + 3.f;
    u_bits = __float_as_int(u);
    v_bits = __float_as_int(fmaf((hi - (u - 3.f)) + lo, 0x1p44f, EX_ROUND));
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

// Eight logits as they stand in memory.
template <int TYPE>
struct Raw {
    uint4 v[TYPE == MTP_F32 ? 2 : 1];
};
template <int TYPE>
__device__ __forceinline__ Raw<TYPE> no_logits() {  // -inf
    constexpr uint32_t NONE = TYPE == MTP_F32 ? 0xff800000u : TYPE == MTP_BF16 ? 0xff80ff80u : 0xfc00fc00u;
    Raw<TYPE> r;
    r.v[0] = make_uint4(NONE, NONE, NONE, NONE);
    if constexpr (TYPE == MTP_F32) r.v[1] = r.v[0];
    return r;
}
// Tokens first .. first + 7 at the row's ends, or at any place, one by one.
template <int TYPE>
__device__ __noinline__ Raw<TYPE> fetch_each(const typename Logit<TYPE>::type* x, int first, int vocab) {
    Raw<TYPE> r;
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool in = first + i >= 0 && first + i < vocab;
        if constexpr (TYPE == MTP_F32)
            w[i] = in ? __float_as_uint(x[first + i]) : 0xff800000u;
        else
            w[i] = in ? (uint32_t)x[first + i] : TYPE == MTP_BF16 ? 0xff80u : 0xfc00u;
    }
    if constexpr (TYPE == MTP_F32) {
        r.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
        r.v[1] = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
        r.v[0] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    }
    return r;
}
template <int TYPE>
__device__ __forceinline__ void decode(const Raw<TYPE>& r, float (&v)[8]) {
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
// A row of logits.  Its blocks begin at the 16-byte boundary at or before the row: place j is token j - shift.
template <int TYPE>
struct Row {
    const typename Logit<TYPE>::type* x;
    int shift, vocab;
    __device__ __forceinline__ Row(const void* base, long long row, long long stride, int n) : vocab(n) {
        x = static_cast<const typename Logit<TYPE>::type*>(base) + row * stride;
        shift = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(*x));
    }
    __device__ __forceinline__ bool in(int token) const { return token >= 0 && token < vocab; }
    __device__ __forceinline__ float at(int token) const { return tame(Logit<TYPE>::get(x + token)); }
    // places j .. j + 7 (j a multiple of 8); -inf outside the row, no token's
    __device__ __forceinline__ Raw<TYPE> fetch(int j) const {
        const int first = j - shift;
        if (!(first >= 0 && first + 8 <= vocab)) return fetch_each<TYPE>(x, first, vocab);
        Raw<TYPE> r;
        r.v[0] = *reinterpret_cast<const uint4*>(x + first);
        if constexpr (TYPE == MTP_F32) r.v[1] = *reinterpret_cast<const uint4*>(x + first + 4);
        return r;
    }
};
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
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
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(__float_as_uint(s.top)), "r"(__float_as_uint(s.sum)), "r"(s.arg), "r"(0)
                 : "memory");
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

// A lane's part of the places [from, to) of a row, with what values that are not finite count as.
template <int TYPE>
__device__ __noinline__ Stat tame_stat(const Row<TYPE>& row, int from, int to, float c) {
    Stat s{-VF_HUGE, 0.f, INT_MAX};
#pragma unroll 1
    for (int j = from + (threadIdx.x & 31); j < to; j += 32) {
        const int token = j - row.shift;
        if (!row.in(token)) continue;
        const float x = row.at(token), top = fmaxf(s.top, x);
        s.sum = s.sum * ex2((s.top - top) * c) + ex2((x - top) * c);
        if (x > s.top || s.arg == INT_MAX) s.arg = token;
        s.top = top;
    }
    return s;
}
// u q(d) < p(d) in 64 bits: x, y the logits, sums in 2^-44 (of q: 0, all of it is on d).
__device__ __noinline__ bool near_kept(float u, float x, float top, long long sum, float y, float y_top, long long y_sum, float t) {
    const double c = 1.4426950408889634 / (double)t;
    double q = 1.0;
    if (y_sum > 0) q = exp2(((double)y - (double)y_top) * c) / ((double)y_sum * 0x1p-44);
    return (double)u * q < exp2(((double)x - (double)top) * c) / ((double)sum * 0x1p-44);
}

// A window's weights of one distribution in shared memory, by places: 45 bits each, the lowest 13 of them apart.
struct Held {
    uint32_t hi, lo;  // addresses: words, halfwords
    // places i .. i + 7 of the window (i a multiple of 8)
    __device__ __forceinline__ void put(int i, const long long (&w)[8]) const {
        uint32_t x[8], y[4];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = (uint32_t)(w[k] >> 13);
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = ((uint32_t)w[2 * k] & 8191) | ((uint32_t)w[2 * k + 1] & 8191) << 16;
#pragma unroll
        for (int k = 0; k < 8; k += 4)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(hi + (i + k) * 4), "r"(x[k]), "r"(x[k + 1]), "r"(x[k + 2]), "r"(x[k + 3]) : "memory");
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(lo + i * 2), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
    }
    __device__ __forceinline__ unsigned long long get(int i) const {
        uint32_t x;
        uint16_t y;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(hi + i * 4) : "memory");
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(y) : "r"(lo + i * 2) : "memory");
        return (unsigned long long)x << 13 | y;
    }
};
// Weights of tokens [from, to) of a row; returns this thread's sum.  One body for all calls: inlined at each, the kernel's
// instructions did not stay in the cache.
template <int TYPE, int NT>
__device__ __noinline__ long long hold_weights(const Row<TYPE> row, const Exponent e, uint32_t table, const Held held, int from, int to) {
    long long sum = 0;
    const int g0 = (from + row.shift) >> 3;  // the window's first eight places
    int g = g0 + threadIdx.x;
    Raw<TYPE> next = row.fetch(g * 8);
#pragma unroll 1
    for (; g * 8 - row.shift < to; g += NT) {
        const int first = g * 8 - row.shift;
        float x[8];
        decode<TYPE>(next, x);
        if (first + 8 * NT < to) next = row.fetch((g + NT) * 8);  // on its way
        const bool all = first >= from && first + 8 <= min(to, row.vocab);
        int su = 0, sv = 0;
        long long w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            int u, v;
            ex_fixed(x[i], e, table, u, v);
            u -= EX_U;
            v -= EX_V;
            // (another window's, or none's, where -inf may count as a number)
            if (!all && (!row.in(first + i) || first + i < from || first + i >= to)) u = v = 0;
            su += u;
            sv += v;
            w[i] = ((long long)u << 22) + v;
        }
        held.put((g - g0) * 8, w);
        sum += ((long long)su << 22) + sv;
    }
    return sum;
}

// How the weights of a draw are made.
enum DrawMode { DRAW_TARGET, DRAW_WITHOUT, DRAW_REST };  // p; p but for the drafted token; max(p - q, 0)

// Grid (slots * ctas).
template <int TYPE, int NT>
__global__ void __launch_bounds__(NT, 512 / NT) draft_verify_kernel(const __grid_constant__ DraftArgs p) {
    constexpr int WARPS = NT / 32, WINDOW = VF_WINDOW<NT>;
    extern __shared__ __align__(16) unsigned char vf_sm[];
    __shared__ int state[VF_MAX_NEW], fed[VF_MAX_NEW];  // of each draft: kept (2: near), the token
    __shared__ float numbers[VF_MAX_NEW];               // the rows' numbers for a draw
    __shared__ long long warp_total[2][WARPS], word[2][2][VF_MAX_CLUSTER];
    __shared__ int s_block;
    __shared__ long long s_before, s_at;
    const mtp_draft_verify_args& a = p.a;
    ExEntry* table = reinterpret_cast<ExEntry*>(vf_sm);
    Stat* stat = reinterpret_cast<Stat*>(vf_sm + sizeof(ExTable));  // [2 max_new], of rows
    Stat* parts = stat + 2 * a.max_new;                             // [2 max_new + warps], of the warps' parts of them
    Stat* gather = parts + 2 * a.max_new + WARPS;                   // [ctas][2 max_new]
    long long* block_sum = reinterpret_cast<long long*>(gather + p.ctas * 2 * a.max_new);  // [blocks]
    const int window = min(p.blocks, WINDOW) * VF_BLOCK;
    const uint32_t table_at = smem_addr(table), held_at = (smem_addr(block_sum + p.blocks) + 15) & ~15u;
    const int room = window + 16;  // places of a window's tokens, in eights
    const Held held_p{held_at, held_at + 8 * room}, held_q{held_at + 4 * room, held_at + 10 * room};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, C = p.ctas, slot = blockIdx.x / C, rank = blockIdx.x - slot * C;
    constexpr int ITEM = VF_ITEM<TYPE>;
    const int V = a.vocab;
    pdl_launch_dependents();
    if (C > 1) cluster_arrive_relaxed();  // (before the first push every CTA is there)
#pragma unroll 1
    for (int i = tid; i < EX_STEPS; i += NT) table[i] = ex_table.e[i];
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
    const float T = a.temperature ? a.temperature[slot] : 1.f;
    const bool bad = r0 < 0 || n < 0 || end > a.rows || n > a.max_new || len < n ||
                     (a.block_table && len > (long long)a.bt_stride << p.shift);
    int* out = a.out_tokens + (long long)slot * a.max_new;
    if (bad || n == 0) {  // (the whole cluster)
        if (C > 1) cluster_wait();
        if (rank == 0) {
#pragma unroll 1
            for (int i = tid; i < a.max_new; i += NT) out[i] = -1;
            if (tid == 0) {
                a.out_counts[slot] = 0;
                a.out_kv_lens[slot] = len;
                if (a.out_done) a.out_done[slot] = 0;
                if (bad && a.err_word) atomicOr(a.err_word, ERR_BOUNDS);
            }
        }
        return;
    }
    const bool greedy = !(T > 0.f), drafter = a.draft_logits && !greedy;
    // c = log2 e / T as hi + lo.  (All in 32 bits: 64-bit operations of a CTA's threads take microseconds.)
    const float t_tame = fminf(fmaxf(T, 1e-30f), 1e30f), cf = 1.44269502f / t_tame;
    const float c_lo = (fmaf(-cf, t_tame, 1.44269502f) + 1.92596299e-8f) / t_tame;
    const int b0 = rank * p.blocks;  // this CTA's blocks of every row (of places there, of tokens below)

    // ---- 1: every row's largest logit and sum ----
    const int tasks = n + (drafter ? n - 1 : 0), items = (p.blocks + ITEM - 1) / ITEM, total = tasks * items;
    auto row_of = [&](int task) {
        return task < n ? Row<TYPE>(a.logits, r0 + task, a.logits_stride, V) : Row<TYPE>(a.draft_logits, r0 + task - n, a.draft_stride, V);
    };
    // what the drafts are judged by, on its way
    int draft = -1;
    float draft_u = 0.f, draft_x = 0.f, draft_y = 0.f;
    if (tid < n) numbers[tid] = a.uniforms[2 * (r0 + tid) + 1];
    if (tid < n - 1) {
        fed[tid] = draft = a.tokens[r0 + 1 + tid];
        draft_u = a.uniforms[2 * (r0 + tid)];
        if (draft >= 0 && draft < V) {
            draft_x = row_of(tid).at(draft);
            if (drafter) draft_y = row_of(n + tid).at(draft);
        }
    }
    auto first_item = [&](int w) { return (int)((long long)total * w / WARPS); };
#pragma unroll 1
    for (int it = first_item(warp), stop = first_item(warp + 1); it < stop;) {
        const int task = it / items, from = it, to = min(stop, (task + 1) * items);  // items [from, to) of a row
        const Row<TYPE> row = row_of(task);
        Stat s{-VF_HUGE, 0.f, INT_MAX};
        Raw<TYPE> raw[ITEM], next[ITEM];
#pragma unroll 1
        for (int at = from - 1; at < to; ++at) {
            // the next item's logits are on their way (the first one's: nothing else is there to do)
            const int block = b0 + (at - task * items) * ITEM, stop_block = at + 1 < to ? min(b0 + p.blocks, block + 2 * ITEM) : 0;
#pragma unroll
            for (int k = 0; k < ITEM; ++k) {
                raw[k] = next[k];
                next[k] = block + ITEM + k < stop_block ? row.fetch((block + ITEM + k) * VF_BLOCK + lane * 8) : no_logits<TYPE>();
            }
            if (at < from) continue;
            float x[ITEM][8], top = s.top;
#pragma unroll
            for (int k = 0; k < ITEM; ++k) {
                decode<TYPE>(raw[k], x[k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, x[k][i]);
            }
            if (greedy) {
                if (top > s.top || s.arg == INT_MAX) {
                    int arg = INT_MAX;
#pragma unroll
                    for (int k = ITEM - 1; k >= 0; --k)
#pragma unroll
                        for (int i = 7; i >= 0; --i) arg = x[k][i] == top ? (k << 8) + i : arg;
                    if (arg != INT_MAX) s.arg = block * VF_BLOCK + lane * 8 - row.shift + arg;
                }
            } else {
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                const float low = -top * cf;  // (its rounding, 2^-24 of it, is all of the sum's: the comparison below allows for it)
#pragma unroll
                for (int k = 0; k < ITEM; ++k)
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const float2 z = fma2(make_float2(x[k][i], x[k][i + 1]), make_float2(cf, cf), make_float2(low, low));
                        sum[i >> 1 & 1] = add2(sum[i >> 1 & 1], make_float2(ex2(z.x), ex2(z.y)));
                    }
                s.sum = fmaf(s.sum, ex2((s.top - top) * cf), (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y));
            }
            s.top = top;
        }
        it = to;
        const float most = warp_max(s.top);
        const int first = (b0 + (from - task * items) * ITEM) * VF_BLOCK, past = min(b0 + p.blocks, b0 + (to - task * items) * ITEM) * VF_BLOCK;
        if (most == -VF_HUGE) {  // nothing above what -infinity counts as: its tokens, if there are any, alike
            const int token = max(0, first - row.shift), tokens = max(0, min(V, past - row.shift) - token);
            s = Stat{-VF_HUGE, lane == 0 ? (float)tokens : 0.f, tokens > 0 ? token : INT_MAX};
        } else if (!__all_sync(FULL_MASK, s.sum >= 0.f) || !(most < VF_HUGE)) {
            // values that are not finite show in the sum or the largest: the row's part once more, with care
            s = tame_stat<TYPE>(row, first, past, cf);
        }
        s = merge(s, cf);
        if (lane == 0) parts[task + warp] = s;
    }
    __syncthreads();
    if (C > 1) cluster_wait();
#pragma unroll 1
    for (int task = warp; task < tasks; task += WARPS) {  // a lane per warp's part, then per CTA
        const bool has = lane < WARPS && max(first_item(lane), task * items) < min(first_item(lane + 1), (task + 1) * items);
        const Stat s = merge(has ? parts[task + lane] : Stat{-VF_HUGE, 0.f, INT_MAX}, cf);
        if (lane < C) push(&gather[rank * 2 * a.max_new + task], lane, s);
    }
    team();
#pragma unroll 1
    for (int task = warp; task < tasks; task += WARPS) {
        Stat s = merge(lane < C ? gather[lane * 2 * a.max_new + task] : Stat{-VF_HUGE, 0.f, INT_MAX}, cf);
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
                const float size = fabsf(stat[tid].top) + (drafter ? fabsf(stat[n + tid].top) : 0.f);
                // too near for 32 bits (a sum's error from its exponents: 2^-24 ln 2 of the largest, doubled)
                if (!(fabsf(l - r) > (VF_NEAR + 0x1p-23f * size * cf) * big) || big < 1e-25f) keep = 2;
            }
        }
        state[tid] = keep;
    }
    __syncthreads();

    int turn = 0;  // which of the words the next sum over the CTAs uses
    // sums over the cluster of the warps' totals, and the first one's over the CTAs before this one
    auto all_sums = [&](long long (&all)[2], long long& before) {
        __syncthreads();
        if (warp < 2) {
            long long t = lane < WARPS ? warp_total[warp][lane] : 0;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(FULL_MASK, t, o);  // (in all lanes: up to 16 push it)
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
    int kept = 0, token = V;  // V: not this CTA's
    bool cut = false;
    if (tid == 0) s_block = -1;
    const int t0 = b0 * VF_BLOCK, t1 = t0 + p.blocks * VF_BLOCK;  // this CTA's tokens
#pragma unroll 1
    for (bool drawn = false; !drawn;) {
#pragma unroll 1
        for (; !cut && kept < n - 1 && state[kept] == 1; ++kept) cut = fed[kept] == a.eos_id;
        if (cut) break;
        if (greedy) {
            if (rank == 0) token = stat[kept].arg;
            break;
        }
        // ---- 3: the row that a token is drawn behind, or that has to be looked at in 64 bits ----
        const bool more = kept < n - 1, near = more && state[kept] == 2;
        const int other = more && drafter ? n + kept : kept;
        DrawMode mode = !more ? DRAW_TARGET : drafter ? DRAW_REST : DRAW_WITHOUT;
        const Row<TYPE> t = row_of(kept), d = row_of(other);
        const Exponent zp = make_exponent(stat[kept].top, cf, c_lo);
        const Exponent zq = make_exponent(stat[other].top, cf, c_lo);
        const int without = more ? fed[kept] : -1;
        unsigned long long sp = 0, sq = 0;  // sums, shifted up: weights times the other one's are in the same units
        long long noise = 0;                // what rounding may leave of p - q, where they are the same
        int held_from = -1;                 // first token of the window that is held
        auto hold = [&](int from, long long (&sum)[2]) {
            __syncthreads();  // (another window may still be read)
            sum[0] += hold_weights<TYPE, NT>(t, zp, table_at, held_p, from, min(from + window, t1));
            if (mode == DRAW_REST) sum[1] += hold_weights<TYPE, NT>(d, zq, table_at, held_q, from, min(from + window, t1));
            held_from = from;
        };
        auto weight = [&](int token) {  // of the window that is held
            long long w = (long long)held_p.get(token + t.shift - ((held_from + t.shift) & ~7));
            if (mode == DRAW_REST) {
                const unsigned long long q = held_q.get(token + d.shift - ((held_from + d.shift) & ~7));
                w = max((long long)__umul64hi(w, sq) - (long long)__umul64hi(q, sp), 0ll);
            }
            if (mode == DRAW_WITHOUT && token == without) w = 0;
            return w;
        };
        // 0: both sums, where they are needed; 1: the weights' sums of blocks; 2: the token
        long long at = 0;
#pragma unroll 1
        for (int pass = near || mode == DRAW_REST ? 0 : 1; !drawn;) {
            long long total[2] = {0, 0}, again[2];  // again: of weights that were added up before
            if (pass == 2) {
                const int k = s_block;
                if (k >= 0) {  // (the whole CTA)
                    const int from = t0 + k / WINDOW * WINDOW * VF_BLOCK, first = t0 + k * VF_BLOCK + lane * 8;
                    if (held_from != from) hold(from, again);
                    __syncthreads();
                    if (warp == 0) {
                        long long w[8], s = 0;
#pragma unroll
                        for (int i = 0; i < 8; ++i) s += w[i] = weight(first + i);
                        s = warp_scan(s) + s_before - s;
                        int found = V;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            s += w[i];
                            if (s > at && found == V) found = first + i;
                        }
                        token = __reduce_min_sync(FULL_MASK, found);
                    }
                }
                drawn = true;
                break;
            }
#pragma unroll 1
            for (int from = t0; from < t1; from += window) {
                if (pass == 0) {
                    hold(from, total);
                    continue;
                }
                if (held_from != from) hold(from, again);
                __syncthreads();
                const int blocks = (min(from + window, t1) - from) / VF_BLOCK;
                long long sum = 0;
#pragma unroll 1
                for (int k = warp; k < blocks; k += WARPS) {
                    long long s = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) s += weight(from + k * VF_BLOCK + i * 32 + lane);
                    // (s < 2^48: two parts whose sums over a warp have 32 bits)
                    const uint32_t lo = __reduce_add_sync(FULL_MASK, (uint32_t)s & ((1u << 26) - 1)), hi = __reduce_add_sync(FULL_MASK, (uint32_t)(s >> 26));
                    s = ((long long)hi << 26) + lo;
                    if (lane == 0) block_sum[(from - t0) / VF_BLOCK + k] = s;
                    sum += s;
                }
                total[0] += lane == 0 ? sum : 0;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                total[0] += __shfl_xor_sync(FULL_MASK, total[0], o);
                total[1] += __shfl_xor_sync(FULL_MASK, total[1], o);
            }
            if (lane == 0) {
                warp_total[0][warp] = total[0];
                warp_total[1][warp] = total[1];
            }
            long long all[2], before;
            all_sums(all, before);
            if (pass == 0) {
                if (near) {
                    if (tid == 0)
                        state[kept] = near_kept(unit(a.uniforms[2 * (r0 + kept)]), t.at(without), stat[kept].top, all[0],
                                                d.at(without), stat[other].top, drafter ? all[1] : 0, t_tame);
                    __syncthreads();
                    if (state[kept] == 1) break;  // on to the next draft
                }
                const int up = __clzll(max(all[0], all[1]));
                sp = (unsigned long long)all[0] << up;
                sq = (unsigned long long)all[1] << up;
                // (a weight errs by 2^-33 of itself at most, a share by twice that; half of what two shares differ by is above 0)
                noise = (long long)(__umul64hi(all[0], sq) >> 32);
                pass = 1;
            } else if (all[0] <= noise && mode != DRAW_TARGET) {  // nothing is left of p: p
                mode = DRAW_TARGET;
            } else {
                // the token's weight covers this place
                if (tid == 0) s_at = min((long long)((double)unit(numbers[kept]) * (double)all[0]), all[0] - 1) - before;
                __syncthreads();
                at = s_at;
                if (warp == 0 && at >= 0) {
                    long long base = 0;
#pragma unroll 1
                    for (int k0 = 0; k0 < p.blocks; k0 += 32) {
                        const int k = k0 + lane;
                        const long long s = k < p.blocks ? block_sum[k] : 0, x = base + warp_scan(s);
                        if (x > at && x - s <= at) {
                            s_block = k;
                            s_before = x - s;
                        }
                        base = __shfl_sync(FULL_MASK, x, 31);
                    }
                }
                __syncthreads();
                pass = 2;
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
#pragma unroll 1
        for (int i = tid; i < a.max_new; i += NT)
            if (i != kept || cut) out[i] = i < kept ? fed[i] : -1;
        if (tid == 0) {
            a.out_counts[slot] = cut ? kept : kept + 1;
            a.out_kv_lens[slot] = after;
            if (cut && a.out_done) a.out_done[slot] = 1;
        }
        if (a.block_table) {
            const int mask = (1 << p.shift) - 1, from = (after + mask) >> p.shift, to = (len + mask) >> p.shift;
#pragma unroll 1
            for (int i = from + tid; i < to; i += NT) {
                int* entry = a.block_table + (long long)slot * a.bt_stride + i;
                const int page = *entry;
                const bool there = page >= 0 && page < a.n_pages;
                *entry = -1;
                if (there && atomicSub(a.page_refs + page, 1) >= 1) continue;
                if (there) atomicAdd(a.page_refs + page, 1);  // it was free already
                if (a.err_word) atomicOr(a.err_word, ERR_BOUNDS);
            }
        }
    }
}

cudaError_t allow_wide_cluster(const void* kernel) {  // (setting it again changes nothing)
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
}
template <int TYPE, int NT>
cudaError_t launch_threads(const DraftArgs& p, cudaStream_t s) {
    const size_t stats = 2 * p.a.max_new * (2 + p.ctas) + NT / 32, window = (size_t)std::min(p.blocks, VF_WINDOW<NT>) * VF_BLOCK;
    const size_t smem = sizeof(ExTable) + stats * sizeof(Stat) + p.blocks * sizeof(long long) + 16 + (window + 16) * 12;
    if (p.ctas > 8) {
        const cudaError_t e = allow_wide_cluster(reinterpret_cast<const void*>(draft_verify_kernel<TYPE, NT>));
        if (e != cudaSuccess) return e;
    }
    return launch(draft_verify_kernel<TYPE, NT>, p.a.slots * p.ctas, NT, smem, p.ctas, s, p);
}
template <int TYPE>
cudaError_t launch_verify(const DraftArgs& p, bool wide, cudaStream_t s) {
    return wide ? launch_threads<TYPE, 512>(p, s) : launch_threads<TYPE, 256>(p, s);
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
        // A slot's CTAs: as many as there are SMs for, as long as their parts of a row are a few blocks.  32 slots of 48001, us: 4 CTAs of 512
        // threads 30; 8 of 256, two an SM, 34, of 512 40.
        int ctas = 1;
        while (ctas < VF_MAX_CLUSTER && (long long)a->slots * ctas * 2 <= sms && a->vocab / (ctas * 2) >= VF_BLOCK * 4) ctas *= 2;
        // CTAs of 512 threads, an SM each, if all run at once.  One slot of 32003, us: 14.1, of 256 threads 14.5; 128 slots of 9000 26.1 and 57.
        // Wide clusters that the SMs hold side by side leave some of them over, 17 of 8 CTAs: 9000 19.0, of 256 threads, two an SM, 15.8; 8 of 16:
        // 48001 21.3 and 19.8.  More slots than SMs: long rows want the threads (200 of 48001 170 and 262, of 9000 37 and 61), short ones the two
        // slots an SM (200 of 4000 22.1 and 21.1, of 1025 18.1 and 14.1).
        const bool wide = a->slots > sms ? a->vocab > 8192 : ctas < 8 || a->slots * ctas * 4 <= sms * 3;
        const int most = 16 / size - 1;  // places before a row's first token
        const int blocks = (a->vocab + most + VF_BLOCK - 1) / VF_BLOCK;
        const DraftArgs p{*a, a->block_table ? log2_of(a->page_size) : 0, ctas, (blocks + ctas - 1) / ctas};
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        e = a->logits_dtype == MTP_F32    ? launch_verify<MTP_F32>(p, wide, s)
            : a->logits_dtype == MTP_BF16 ? launch_verify<MTP_BF16>(p, wide, s)
                                          : launch_verify<MTP_F16>(p, wide, s);
        return cuda_status(e, "draft_verify");
    });
}

}  // extern "C"
