// rotary.cu -- rotary positions of a step's queries and keys, and keys and values into the
// paged cache (mtp_rotary_append); the pairs' turns per position (mtp_rotary_turns).
//
//   (a, b) -> g (a cos t - b sin t, a sin t + b cos t),  t = 2 pi position * turns_i,
//
// for the pairs i of a head's first rot_dim elements: a and b are elements i and i + rot_dim / 2
// (halves) or 2 i and 2 i + 1 (pairs).  The rest of the head, and the values, are only rounded.
//
// A pair's turns per position are a 64-bit fraction of 2^64: the product with the position, modulo
// 2^64, is the angle modulo whole turns, exactly.  What is left of the error is half the fraction's last
// place times the position, 2^-34 of a turn at most (the fractions are made in twice fp64's precision: fp64's 53 bits
// would be off by 2^-24 of a turn at position 2^31), and the rounding of the 32 highest bits to fp32.  (fp32 products position * frequency are off by up to 0.03 radians at position 1,000,000; fp64's sine
// and cosine would be most of a call.)
//
// Bound by memory: every element is read and written once.  A CTA takes a few rows: its threads
// ask for their elements, make the rows' sines and cosines in shared memory meanwhile (a pair's
// serve all heads), and turn.  14592 rows of 16 heads of 64 from fp32: 269 MB in 41.6 us, 6.5 TB/s; four pieces a thread
// at once 48.0 us, two and no more registers than four CTAs of an SM have 41.6 (three CTAs 43.0, rows for
// one batch or four of those 47.7, 48.2).  A step's 32 rows are latency, 2.7 us.  Halves that are no multiple of 8 long have
// their partners loaded one by one: 14592 such rows with 40 of 64 elements turned take 69 us.
#include <algorithm>
#include <climits>
#include <cmath>

#include "serving.cuh"

namespace mtp {
namespace {

constexpr int RO_THREADS = 256, RO_UNROLL = 2, RO_BATCHES = 2;

// How a head is cut into the threads' pieces.  HALVES and PAIRS: 16 elements, the two of every pair among them; ANY: 8
// (halves that are no multiple of 8 long: the partners are loaded one by one).
enum RotaryPieces { PIECES_HALVES, PIECES_PAIRS, PIECES_ANY };

struct RotaryArgs {
    mtp_rotary_append_args a;
    int shift;            // page_size = 1 << shift
    int cta_rows;         // rows of a CTA
    unsigned pieces, hp;  // pieces of a row, of a head
};

template <class T, int SRC>
struct Source;
template <class T>
struct Source<T, MTP_F32> {
    using type = float;
    struct Vec {
        float4 x, y;
    };
    static __device__ __forceinline__ float one(const float* p) { return *p; }
    template <bool VECTOR>
    static __device__ __forceinline__ Vec load(const float* p) {
        if constexpr (VECTOR) return Vec{*reinterpret_cast<const float4*>(p), *(reinterpret_cast<const float4*>(p) + 1)};
        return Vec{make_float4(p[0], p[1], p[2], p[3]), make_float4(p[4], p[5], p[6], p[7])};
    }
    static __device__ __forceinline__ void floats(const Vec& v, float (&f)[8]) {
        f[0] = v.x.x; f[1] = v.x.y; f[2] = v.x.z; f[3] = v.x.w;
        f[4] = v.y.x; f[5] = v.y.y; f[6] = v.y.z; f[7] = v.y.w;
    }
    static __device__ __forceinline__ uint4 rounded(const Vec& v) {
        return make_uint4(T::pack(v.x.x, v.x.y), T::pack(v.x.z, v.x.w), T::pack(v.y.x, v.y.y), T::pack(v.y.z, v.y.w));
    }
};
template <class T>
struct Source<T, MTP_BF16> {  // the pool's own type
    using type = uint16_t;
    using Vec = uint4;
    static __device__ __forceinline__ float one(const uint16_t* p) { return T::to_float(*p); }
    template <bool VECTOR>
    static __device__ __forceinline__ Vec load(const uint16_t* p) {
        if constexpr (VECTOR) return *reinterpret_cast<const uint4*>(p);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (uint32_t)p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ void floats(const Vec& v, float (&f)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = T::to_float((uint16_t)w[i]);
            f[2 * i + 1] = T::to_float((uint16_t)(w[i] >> 16));
        }
    }
    static __device__ __forceinline__ uint4 rounded(const Vec& v) { return v; }
};

__device__ __forceinline__ void store8(uint16_t* to, const uint4& v, bool vector) {
    if (vector) {
        *reinterpret_cast<uint4*>(to) = v;
        return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        to[2 * i] = (uint16_t)w[i];
        to[2 * i + 1] = (uint16_t)(w[i] >> 16);
    }
}
template <class T>
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(T::pack(f[0], f[1]), T::pack(f[2], f[3]), T::pack(f[4], f[5]), T::pack(f[6], f[7]));
}

// Where a piece is read and written.  kind: 0 queries, 1 keys, 2 values, -1 none; at: the piece's number in the head.
struct Piece {
    int row, kind, at;
    unsigned head;
    int64_t from, slot;  // element of q, k or v; place in the pool
};

// VECTOR: all three sources' rows on 16-byte boundaries; OUT_VECTOR (a run-time rule): out_q's.
template <class T, int SRC, int PIECES, bool VECTOR>
__global__ void __launch_bounds__(RO_THREADS, 4) rotary_append_kernel(const __grid_constant__ RotaryArgs p, bool out_vector) {
    using S = Source<T, SRC>;
    using E = typename S::type;
    constexpr int VECS = PIECES == PIECES_ANY ? 1 : 2;
    extern __shared__ float2 ro_turns[];  // [cta_rows][rot_dim / 2] cosines and sines
    const mtp_rotary_append_args& a = p.a;
    const int row0 = blockIdx.x * p.cta_rows, rows = min(p.cta_rows, a.rows - row0), half = a.rot_dim >> 1;
    const unsigned total = rows * p.pieces;
    uint16_t *pool = static_cast<uint16_t*>(a.kv_pool), *out_q = static_cast<uint16_t*>(a.out_q);
    pdl_launch_dependents();
    pdl_wait();

    auto piece = [&](unsigned i) {
        Piece x;
        const unsigned r = i / p.pieces, rest = i - r * p.pieces, head = rest / p.hp, c = rest - head * p.hp;
        x.row = row0 + (int)r;
        x.at = (int)c;
        x.slot = 0;
        if (head < (unsigned)a.n_heads) {
            x.kind = 0;
            x.head = head;
            x.from = x.row * a.q_stride + head * a.head_dim;
            return x;
        }
        x.kind = head < (unsigned)(a.n_heads + a.n_kv_heads) ? 1 : 2;
        x.head = head - a.n_heads - (x.kind - 1) * a.n_kv_heads;
        x.from = x.row * (x.kind == 1 ? a.k_stride : a.v_stride) + x.head * a.head_dim;
        x.slot = a.slot_map[x.row];
        return x;
    };
    // the head's first element in out_q or the pool; null: left out
    auto target = [&](const Piece& x) -> uint16_t* {
        if (x.kind == 0) return out_q + x.row * a.out_stride + x.head * a.head_dim;
        const int64_t page = x.slot >> p.shift;
        if (x.slot < 0 || page >= a.n_pages) return nullptr;
        const int64_t block = ((page * a.layers + a.layer) * 2 + (x.kind - 1)) * a.n_kv_heads + x.head;
        return pool + ((block << p.shift) + (x.slot & ((1 << p.shift) - 1))) * a.head_dim;
    };
    // the two places of a piece's eight elements in the head
    auto place = [&](const Piece& x, int v) {
        if (PIECES == PIECES_ANY) return x.at * 8;
        if (PIECES == PIECES_HALVES && x.kind != 2) {
            const int turned = half >> 3;  // pieces of which the first vector's elements have their partners in the second
            if (x.at < turned) return x.at * 8 + v * half;
        }
        return x.at * 16 + v * 8;
    };

    bool first = true;
    for (unsigned i0 = threadIdx.x; first || i0 < total + threadIdx.x; i0 += RO_THREADS * RO_UNROLL) {
        Piece x[RO_UNROLL];
        typename S::Vec v[RO_UNROLL][VECS];
#pragma unroll
        for (int u = 0; u < RO_UNROLL; ++u) {
            const unsigned i = i0 + u * RO_THREADS;
            x[u].kind = -1;
            if (i >= total) continue;
            x[u] = piece(i);
            const E* src = static_cast<const E*>(x[u].kind == 0 ? a.q : x[u].kind == 1 ? a.k : a.v) + x[u].from;
#pragma unroll
            for (int e = 0; e < VECS; ++e) v[u][e] = S::template load<VECTOR>(src + place(x[u], e));
        }
        if (first) {
            for (int j = threadIdx.x; j < rows * half; j += RO_THREADS) {
                const int r = j / half, pair = j - r * half;
                const uint64_t turn = (uint64_t)(int64_t)a.positions[row0 + r] * a.turns[pair];
                float s, c;
                sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &s, &c);
                ro_turns[j] = make_float2(a.gain * c, a.gain * s);
            }
            __syncthreads();
            first = false;
        }
#pragma unroll
        for (int u = 0; u < RO_UNROLL; ++u) {
            if (x[u].kind < 0) continue;
            uint16_t* to = target(x[u]);
            if (!to) continue;
            const bool vector = x[u].kind != 0 || out_vector;
            const float2* cs = ro_turns + (x[u].row - row0) * half;
            uint4 y[VECS];
#pragma unroll
            for (int e = 0; e < VECS; ++e) y[e] = S::rounded(v[u][e]);
            if (x[u].kind != 2) {
                if constexpr (PIECES == PIECES_HALVES) {
                    if (x[u].at < half >> 3) {
                        float lo[8], hi[8], f[8], g[8];
                        S::floats(v[u][0], lo);
                        S::floats(v[u][1], hi);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float2 t = cs[x[u].at * 8 + e];
                            f[e] = fmaf(lo[e], t.x, -(hi[e] * t.y));
                            g[e] = fmaf(lo[e], t.y, hi[e] * t.x);
                        }
                        y[0] = pack8<T>(f);
                        y[1] = pack8<T>(g);
                    }
                } else {
                    const bool pairs = PIECES == PIECES_PAIRS || a.layout == MTP_ROTARY_PAIRS;
#pragma unroll
                    for (int e = 0; e < VECS; ++e) {
                        const int at = place(x[u], e);
                        if (at >= a.rot_dim) continue;
                        float f[8], g[8];
                        S::floats(v[u][e], f);
                        if (pairs) {
#pragma unroll
                            for (int n = 0; n < 8; n += 2) {
                                const bool in = at + n < a.rot_dim;
                                const float2 t = cs[in ? (at + n) >> 1 : 0];
                                g[n] = in ? fmaf(f[n], t.x, -(f[n + 1] * t.y)) : f[n];
                                g[n + 1] = in ? fmaf(f[n], t.y, f[n + 1] * t.x) : f[n + 1];
                            }
                        } else {
                            const E* src = static_cast<const E*>(x[u].kind == 0 ? a.q : a.k) + x[u].from;
#pragma unroll
                            for (int n = 0; n < 8; ++n) {
                                const int i = at + n;
                                g[n] = f[n];
                                if (i >= a.rot_dim) continue;
                                const bool low = i < half;
                                const float other = S::one(src + (low ? i + half : i - half));
                                const float2 t = cs[low ? i : i - half];
                                g[n] = low ? fmaf(f[n], t.x, -(other * t.y)) : fmaf(other, t.y, f[n] * t.x);
                            }
                        }
                        const uint4 z = pack8<T>(g);
                        if (at + 8 <= a.rot_dim) {
                            y[e] = z;
                        } else {  // what is not turned stays bit by bit
                            const uint32_t w[4] = {z.x, z.y, z.z, z.w};
                            uint32_t b[4] = {y[e].x, y[e].y, y[e].z, y[e].w};
#pragma unroll
                            for (int n = 0; n < 4; ++n)
                                if (at + 2 * n < a.rot_dim) b[n] = w[n];
                            y[e] = make_uint4(b[0], b[1], b[2], b[3]);
                        }
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < VECS; ++e) store8(to + place(x[u], e), y[e], vector);
        }
    }
}

template <class T, int SRC, int PIECES>
cudaError_t launch_pieces(const RotaryArgs& p, bool vector, bool out_vector, cudaStream_t s) {
    const int grid = (p.a.rows + p.cta_rows - 1) / p.cta_rows;
    const size_t smem = (size_t)p.cta_rows * (p.a.rot_dim / 2) * sizeof(float2);
    return vector ? launch_ex(rotary_append_kernel<T, SRC, PIECES, true>, dim3(grid), RO_THREADS, smem, s, 1, p, out_vector)
                  : launch_ex(rotary_append_kernel<T, SRC, PIECES, false>, dim3(grid), RO_THREADS, smem, s, 1, p, out_vector);
}
template <class T, int SRC>
cudaError_t launch_rotary(const RotaryArgs& p, bool vector, bool out_vector, cudaStream_t s) {
    if (p.hp * 8 == (unsigned)p.a.head_dim) return launch_pieces<T, SRC, PIECES_ANY>(p, vector, out_vector, s);
    return p.a.layout == MTP_ROTARY_HALVES ? launch_pieces<T, SRC, PIECES_HALVES>(p, vector, out_vector, s)
                                           : launch_pieces<T, SRC, PIECES_PAIRS>(p, vector, out_vector, s);
}

// ---- the turns, on the host: numbers as sums hi + lo of two fp64, about 100 bits ----

struct Twice {
    double hi, lo;
};
Twice joined(double hi, double lo) {  // |hi| >= |lo|
    const double s = hi + lo;
    return {s, lo - (s - hi)};
}
Twice operator+(Twice x, Twice y) {  // the rounding error of the sum of the first parts, exactly, with the second ones
    const double s = x.hi + y.hi, t = s - x.hi;
    return joined(s, ((x.hi - (s - t)) + (y.hi - t)) + (x.lo + y.lo));
}
Twice operator*(Twice x, Twice y) {
    const double p = x.hi * y.hi;
    return joined(p, std::fma(x.hi, y.hi, -p) + (x.hi * y.lo + x.lo * y.hi));
}
Twice operator-(Twice x) { return {-x.hi, -x.lo}; }
Twice operator/(Twice x, Twice y) {
    const double q = x.hi / y.hi;
    return joined(q, (x + -(y * Twice{q, 0.0})).hi / y.hi);
}
constexpr Twice LN2{0x1.62e42fefa39efp-1, 0x1.abc9e3b39803fp-56}, TURNS{0x1.45f306dc9c883p-3, -0x1.6b01ec5417056p-57};  // TURNS: of a radian, 1 / (2 pi)
// e^x = 2^k (1 + y)^256: y of a 256th of what x has beyond k ln 2, by its series (of at most 0.0014: 12 terms, 2^-140), squared 8 times
Twice exp_twice(Twice x) {
    const double k = std::nearbyint(x.hi / LN2.hi);
    Twice r = x + -(LN2 * Twice{k, 0.0});
    r = {r.hi / 256, r.lo / 256};
    Twice y{0.0, 0.0};
    for (int n = 12; n >= 1; --n) y = r * (y + Twice{1.0, 0.0}) / Twice{(double)n, 0.0};
    for (int i = 0; i < 8; ++i) y = Twice{2 * y.hi, 2 * y.lo} + y * y;
    y = y + Twice{1.0, 0.0};
    return {std::ldexp(y.hi, (int)k), std::ldexp(y.lo, (int)k)};
}
// ln x, x > 0: one step of Newton's method from fp64's, x = 2^e m
Twice log_twice(double x) {
    int e = 0;
    const double m = std::frexp(x, &e), y = std::log(m);
    const Twice d = Twice{m, 0.0} * exp_twice({-y, 0.0}) + Twice{-1.0, 0.0};
    return LN2 * Twice{(double)e, 0.0} + (Twice{y, 0.0} + (d + Twice{-0.5 * d.hi * d.hi, 0.0}));
}

}  // namespace
}  // namespace mtp

using namespace mtp;

extern "C" {

MTP_API int mtp_rotary_turns(int rot_dim, int scaling, double base, double factor, double context, double low,
                             double high, uint64_t* out_turns) {
    return guarded([&]() -> int {
        if (rot_dim < 2 || rot_dim > 256 || rot_dim % 2 || !out_turns)
            return invalid("rotary_turns: rot_dim %d: even, 2 to 256", rot_dim);
        if (scaling < MTP_ROTARY_PLAIN || scaling > MTP_ROTARY_BANDS) return invalid("rotary_turns: scaling %d", scaling);
        if (!(base > 1.0) || !std::isfinite(base)) return invalid("rotary_turns: base %g: above 1", base);
        if (scaling != MTP_ROTARY_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor)))
            return invalid("rotary_turns: factor %g: 1 or more", factor);
        if (scaling == MTP_ROTARY_BASE) {
            if (rot_dim < 4) return invalid("rotary_turns: one pair alone has no base to scale");
            if (!std::isfinite(base * std::pow(factor, rot_dim / (rot_dim - 2.0)))) return invalid("rotary_turns: factor %g", factor);
        }
        if (scaling == MTP_ROTARY_BANDS && !(context > 0.0 && std::isfinite(context) && low < high && std::isfinite(low) && std::isfinite(high)))
            return invalid("rotary_turns: context %g, bands from %g to %g turns", context, low, high);
        const Twice one{1.0, 0.0}, scale{factor, 0.0};
        Twice log_base = log_twice(base);
        if (scaling == MTP_ROTARY_BASE) log_base = log_base + log_twice(factor) * Twice{(double)rot_dim, 0.0} / Twice{rot_dim - 2.0, 0.0};
        for (int i = 0; i < rot_dim / 2; ++i) {
            Twice f = exp_twice(-(log_base * Twice{2.0 * i, 0.0} / Twice{(double)rot_dim, 0.0}));  // radians per position
            if (scaling == MTP_ROTARY_LINEAR) f = f / scale;
            if (scaling == MTP_ROTARY_BANDS) {
                const double about = (context * f.hi * TURNS.hi - low) / (high - low);
                Twice kept{about > 0.5 ? 1.0 : 0.0, 0.0};
                if (about > -0.5 && about < 1.5) {
                    const Twice x = (Twice{context, 0.0} * f * TURNS + Twice{-low, 0.0}) / (Twice{high, 0.0} + Twice{-low, 0.0});
                    kept = x.hi <= 0.0 ? Twice{0.0, 0.0} : x.hi < 1.0 ? x : one;
                }
                f = kept * f + (one + -kept) * f / scale;
            }
            const Twice turns = f * TURNS;
            const double hi = std::ldexp(turns.hi, 64), whole = std::floor(hi);
            out_turns[i] = (uint64_t)whole + (uint64_t)std::llrint((hi - whole) + std::ldexp(turns.lo, 64));
        }
        return MTP_OK;
    });
}

MTP_API int mtp_rotary_append(const mtp_rotary_append_args* a, void* cuda_stream) {
    return guarded([&]() -> int {
        if (!a) return invalid("rotary_append: null arguments");
        if (const int r = check_pool("rotary_append", a->n_pages, a->layers, a->layer, a->n_kv_heads, a->head_dim,
                                     a->page_size))
            return r;
        if (a->rows < 0 || a->n_heads < 1 || a->n_heads > 1024)
            return invalid("rotary_append: rows %d, heads %d", a->rows, a->n_heads);
        if (a->rot_dim < 2 || a->rot_dim % 2 || a->rot_dim > a->head_dim)
            return invalid("rotary_append: rot_dim %d of %d: even, 2 or more", a->rot_dim, a->head_dim);
        if (a->layout != MTP_ROTARY_HALVES && a->layout != MTP_ROTARY_PAIRS)
            return invalid("rotary_append: layout %d", a->layout);
        if (!std::isfinite(a->gain)) return invalid("rotary_append: gain %g", (double)a->gain);
        if ((a->pool_dtype != MTP_BF16 && a->pool_dtype != MTP_F16) ||
            (a->src_dtype != MTP_F32 && a->src_dtype != a->pool_dtype))
            return invalid("rotary_append: src_dtype %d, pool_dtype %d", a->src_dtype, a->pool_dtype);
        const int width = a->n_heads * a->head_dim, kv_width = a->n_kv_heads * a->head_dim;
        if (a->q_stride < width || a->out_stride < width || a->k_stride < kv_width || a->v_stride < kv_width)
            return invalid("rotary_append: row strides %lld, %lld, %lld, %lld below %d, %d, %d, %d", (long long)a->q_stride,
                           (long long)a->k_stride, (long long)a->v_stride, (long long)a->out_stride, width, kv_width, kv_width,
                           width);
        if ((long long)a->rows * (width + 2 * kv_width) > 8ll * INT_MAX) return invalid("rotary_append: rows %d", a->rows);
        if (a->rows == 0) return MTP_OK;
        if (!a->q || !a->k || !a->v || !a->positions || !a->slot_map || !a->turns || !a->kv_pool || !a->out_q)
            return invalid("rotary_append: null pointer");
        if (!aligned16(a->kv_pool)) return invalid("rotary_append: kv_pool must be 16-byte aligned");
        if (a->out_q == a->q) return invalid("rotary_append: out_q needs a buffer of its own");
        const int size = a->src_dtype == MTP_F32 ? 4 : 2;
        if (reinterpret_cast<uintptr_t>(a->q) % size || reinterpret_cast<uintptr_t>(a->k) % size ||
            reinterpret_cast<uintptr_t>(a->v) % size || reinterpret_cast<uintptr_t>(a->out_q) % 2 ||
            reinterpret_cast<uintptr_t>(a->positions) % 4 || reinterpret_cast<uintptr_t>(a->slot_map) % 8 ||
            reinterpret_cast<uintptr_t>(a->turns) % 8)
            return invalid("rotary_append: pointers must be aligned to their elements");
        RotaryArgs p{*a, log2_of(a->page_size), 0, 0, 0};
        // pieces of 16 elements where pairs are whole in them
        const bool wide = a->head_dim % 16 == 0 && (a->layout == MTP_ROTARY_PAIRS || a->rot_dim % 16 == 0);
        p.hp = a->head_dim / (wide ? 16 : 8);
        p.pieces = (a->n_heads + 2 * a->n_kv_heads) * p.hp;
        // a CTA's rows: two batches of its threads', where there are rows enough for every SM
        int dev = 0, sms = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) {
            cudaGetLastError();
            return cuda_status(e, "rotary_append");
        }
        p.cta_rows = (int)std::max(1u, std::min(16u, RO_BATCHES * RO_THREADS * RO_UNROLL / p.pieces));
        p.cta_rows = std::max(1, std::min(p.cta_rows, a->rows / (2 * sms)));
        const bool vector = aligned16(a->q) && aligned16(a->k) && aligned16(a->v) && a->q_stride * size % 16 == 0 &&
                            a->k_stride * size % 16 == 0 && a->v_stride * size % 16 == 0;
        const bool out_vector = aligned16(a->out_q) && a->out_stride % 8 == 0;
        const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
        const bool f32 = a->src_dtype == MTP_F32;
        if (a->pool_dtype == MTP_BF16)
            e = f32 ? launch_rotary<Bf16, MTP_F32>(p, vector, out_vector, s) : launch_rotary<Bf16, MTP_BF16>(p, vector, out_vector, s);
        else
            e = f32 ? launch_rotary<F16, MTP_F32>(p, vector, out_vector, s) : launch_rotary<F16, MTP_BF16>(p, vector, out_vector, s);
        return cuda_status(e, "rotary_append");
    });
}

}  // extern "C"
