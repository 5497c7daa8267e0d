// key_weights_tc.cu -- the kernel of mtp_key_weights for more than 64 rows per slot and key head
// (prompts, chunks), and for more than 16 on keys too few for every SM: tcgen05.
//
//   S^T = K Q^T        128 keys x up to 128 packed rows, fp32 in TMEM
//   w_j += sum_p 2^(c S_jp - l_p)   a key per thread
//
// A CTA has 128 or 512 keys of a slot and key head, which stay in shared memory; the rows that see one
// of them come by, as many tokens as have 128 rows at a time (all heads of a token together, so
// that one tensor-map box is a tile for any number of heads per key head).  A thread's TMEM lane is its
// key: its weights add up in a register, the rows' log-sum-exps are read from shared memory, the
// same one by all lanes, and what a causal or window mask leaves of a tile is a range of columns.  A
// tile's sum starts anew and is added to the key's with compensation, so that thousands of rows cost no
// precision.
// 512 keys: two pairs of tiles of 128, each with a place for S and eight warps, four for each half of the
// columns; a thread has a key of both tiles, so that the log-sum-exps are read once for two.  While one pair
// is summed the tensor cores make the other's.  128 keys: two places, four warps, and two CTAs an SM.
//
// Two chunks of 2000 to 4000 tokens after 6000 to 9000, 32 heads on 8 of 128 dims (540 GFLOP): 400 to 471 us by the GPU, 1150
// TFLOP/s or more, of the measured peak (cuBLAS, 1950) 59 to 69 %, and half of the rate of the exponentials (32 a cycle and
// SM).  (The other figures here are of the GPU that takes 471.)  Without exponentials it takes 387 us, with a quarter of the products 420: neither covers the other's
// latencies whole, and registers for more columns or TMEM for a third place are not there.  128 keys a CTA took
// 614 us: every CTA reads all rows, 7 TB/s out of L2.  25 prompts of 182 to 578 tokens, 16 heads of 64: 36.9 us.
#include <type_traits>

#include "tcgen05.cuh"
#include "weights.cuh"

namespace mtp {
namespace {

constexpr int WT_TILE = 128;
constexpr uint32_t WT_SUB = 128 * 128;  // 128 rows of 128 bytes

// TILES: of 128 keys, that a CTA has.
template <int HD, int TILES>
struct WtLayout {
    static constexpr int STAGES = HD == 64 ? 4 : 2, CTAS = TILES == 1 ? 2 : 1;  // CTAS: of an SM
    // sums: key tiles of a group of warps (they read the rows' log-sum-exps once for all), halves of the columns
    static constexpr int KT = TILES == 1 ? 1 : 2, HALVES = TILES == 1 ? 1 : 2;
    static constexpr int MMA = 4 * TILES, COPY = MMA + 1, THREADS = (COPY + 1) * 32;
    static constexpr uint32_t TM_COLS = TILES == 1 ? 2 * WT_TILE : TILES * WT_TILE;
    static constexpr uint32_t OPER = WT_SUB * (HD / 64);
    static constexpr uint32_t K = 0, Q = TILES * OPER, LSE = Q + STAGES * OPER;  // LSE: [warps][2][columns of a warp] floats
    static constexpr size_t BYTES = 1024 + LSE + 4 * TILES * 2 * (WT_TILE / HALVES) * 4;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tma_box(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            smem_addr(dst)),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_addr(bar))
        : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}
template <class T>
__device__ __forceinline__ uint32_t idesc(int n) {  // f16_idesc's types are bf16; fp16's codes are 0
    const uint32_t d = f16_idesc(WT_TILE, n, false);
    return std::is_same<T, Bf16>::value ? d : d & ~((1u << 7) | (1u << 10));
}

// Grid (group of TILES key tiles and key head, slot, row segment).
template <class T, int HD, int TILES>
__global__ void __launch_bounds__(WtLayout<HD, TILES>::THREADS, WtLayout<HD, TILES>::CTAS)
    key_weights_tc_kernel(const __grid_constant__ WeightsArgs a, const __grid_constant__ CUtensorMap map,
                          const __grid_constant__ CUtensorMap q_map, int q_tma) {
    using L = WtLayout<HD, TILES>;
    constexpr int ST = L::STAGES;
    extern __shared__ unsigned char wt_raw[];
    __shared__ uint64_t k_full, q_full[ST], q_empty[ST], s_full[4], s_empty[4], drain;
    __shared__ uint32_t tmem_base;
    unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(wt_raw) + 1023) & ~(uintptr_t)1023);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int group = blockIdx.x / a.kv_heads, head = blockIdx.x - group * a.kv_heads, slot = blockIdx.y, seg = blockIdx.z;
    pdl_wait();
    bool cut;
    const WeightsSlot s = weights_slot(a, slot, cut);
    if (cut && a.err && blockIdx.x == 0 && seg == 0 && tid == 0) atomicOr(a.err, ERR_BOUNDS);
    const int key0 = group * TILES * WT_TILE, key1 = min(min(s.len, a.keys), key0 + TILES * WT_TILE);
    if (s.n == 0 || key0 >= key1) return;
    // the tokens that see a key of the group, `per` at a time; this segment's tiles of them
    const int2 tokens = seeing(a, s, key0, key1);
    const int per = WT_TILE / a.group, all = (tokens.y - tokens.x + per - 1) / per;
    const int u0 = (int)((long long)all * seg / a.segments), u1 = (int)((long long)all * (seg + 1) / a.segments);
    // of those, the tiles of which some token sees a key of key tile t
    auto range = [&](int t) {
        const int from = key0 + t * WT_TILE, to = min(key1, from + WT_TILE);
        if (from >= to) return make_int2(0, 0);
        const int2 x = seeing(a, s, from, to);
        if (x.x >= x.y) return make_int2(0, 0);
        return make_int2(max(u0, (x.x - tokens.x) / per), min(u1, (x.y - tokens.x + per - 1) / per));
    };
    const int lowest = a.window > 0 ? max(0, s.base - a.window + 1) : 0;  // the first key that some row sees
    float* part = a.part + (((size_t)seg * a.slots + slot) * a.kv_heads + head) * a.width + key0;
    if (u0 >= u1) {
        if (a.segments > 1)
            for (int key = key0 + tid; key < key1; key += L::THREADS)
                if (key >= lowest) part[key - key0] = 0.f;
        return;
    }
    if (warp == L::MMA) {
        tmem_alloc(&tmem_base, L::TM_COLS);
        tmem_relinquish();
    }
    if (tid == 0) {
        mbar_init(&k_full, 1);
        mbar_init(&drain, 1);
        for (int i = 0; i < ST; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&s_empty[i], 4 * L::HALVES);
        }
        fence_barrier_init();
    }
    // rows of a tile past the last token's are zeros
    const int rest = WT_TILE - per * a.group;
    for (int i = tid; i < rest * 8 * (HD / 64) * ST; i += L::THREADS) {
        const int row = per * a.group + i / 8 % rest, half = i / 8 / rest;
        *reinterpret_cast<uint4*>(sm + L::Q + half * WT_SUB + row * 128 + (i & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    // (not before TMEM is there: a kernel behind this one that took it first would wait for this one, which waits for it)
    pdl_launch_dependents();
    auto wait = [&](uint64_t* bar, uint32_t parity) { return __all_sync(FULL_MASK, mbar_wait(bar, parity & 1, a.err)) != 0; };
    // the place of a group of key tiles' c-th tile of rows: one of its own, or (one key tile) the two in turn
    constexpr int KT = L::KT, H = L::HALVES;
    auto place = [](int g, int c) { return TILES == 1 ? c & 1 : g; };
    auto phase = [](int c) { return TILES == 1 ? c >> 1 : c; };
    auto group_range = [&](int g) {  // tiles of rows of which some token sees a key of the group's key tiles
        int2 x = range(g * KT);
        if (KT > 1) {
            const int2 y = range(g * KT + 1);
            x = x.x >= x.y ? y : y.x >= y.y ? x : make_int2(min(x.x, y.x), max(x.y, y.y));
        }
        return x;
    };

    if (warp == L::COPY) {
        // ---- the keys, a lane per page piece, then the rows ----
        const int P = 1 << a.page_shift, box = min(P, WT_TILE), pieces = TILES * WT_TILE / box;
        uint32_t bytes = 0;
        for (int i0 = 0; i0 < pieces; i0 += 32) {
            const bool wanted = i0 + lane < pieces && key0 + (i0 + lane) * box < key1;
            bytes += __popc(__ballot_sync(FULL_MASK, wanted)) * box * 128 * (HD / 64);
        }
        if (lane == 0) mbar_arrive_expect_tx(&k_full, bytes);
        __syncwarp();
        for (int i = lane; i < pieces; i += 32) {
            const int at = key0 + i * box;
            if (at >= key1) break;
            const int page = a.block_table[(size_t)slot * a.bt_stride + (at >> a.page_shift)];
            // (outside the pool: zeros)
            const int block = page >= 0 && page < a.n_pages ? page * a.page_blocks + a.layer_block + head : -1;
            const int row = i * box;  // of the group's
            for (int h = 0; h < HD / 64; ++h)
                tma_box(sm + L::K + (row / WT_TILE) * L::OPER + h * WT_SUB + (row % WT_TILE) * 128, &map, h * 64, at & (P - 1), block, &k_full);
        }
        __syncwarp();
        bool ok = true;
        int n = 0;
        for (; n < u1 - u0; ++n) {
            const int st = n % ST, token = tokens.x + (u0 + n) * per, count = min(per, tokens.y - token);
            if (n >= ST && !(ok = wait(&q_empty[st], n / ST - 1))) break;
            unsigned char* dst = sm + L::Q + st * L::OPER;
            if (q_tma) {
                if (lane == 0) {
                    mbar_arrive_expect_tx(&q_full[st], per * a.group * 128 * (HD / 64));
                    for (int h = 0; h < HD / 64; ++h)
                        tma_box(dst + h * WT_SUB, &q_map, h * 64, head * a.group, s.row0 + token, &q_full[st]);
                }
            } else {  // rows that a tensor map cannot describe: a lane 16 bytes of a row
                for (int i = lane; i < count * a.group * (HD / 8); i += 32) {
                    const int r = i / (HD / 8), c = i - r * (HD / 8), t = r / a.group;
                    const uint16_t* src = a.q + (long long)(s.row0 + token + t) * a.q_stride + (head * a.group + r - t * a.group) * HD + c * 8;
                    uint32_t v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = (uint32_t)src[2 * e] | (uint32_t)src[2 * e + 1] << 16;
                    *reinterpret_cast<uint4*>(dst + (c >> 3) * WT_SUB + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(&q_full[st]);
            }
            __syncwarp();
        }
        if (!ok && lane == 0) {  // what is in flight lands before the CTA leaves
            mbar_wait(&k_full, 0, nullptr);
            for (int i = max(0, n - ST); i < n; ++i) mbar_wait(&q_full[i % ST], (i / ST) & 1, nullptr);
        }
        __syncwarp();
    } else if (warp == L::MMA) {
        if (elect_one()) {
            const uint64_t k = sw128_desc(smem_addr(sm + L::K));
            int2 has[TILES / KT];
            int done[TILES / KT];
#pragma unroll
            for (int g = 0; g < TILES / KT; ++g) {
                has[g] = group_range(g);
                done[g] = 0;
            }
            bool ok = mbar_wait(&k_full, 0, a.err);
            for (int n = 0; ok && n < u1 - u0; ++n) {
                const int st = n % ST, count = min(per, tokens.y - (tokens.x + (u0 + n) * per)) * a.group;
                ok = mbar_wait(&q_full[st], (n / ST) & 1, a.err);
                const uint64_t q = sw128_desc(smem_addr(sm + L::Q + st * L::OPER));
                const uint32_t id = idesc<T>(count == per * a.group ? WT_TILE : (count + 15) & ~15);
#pragma unroll
                for (int g = 0; g < TILES / KT; ++g) {
                    if (!ok || u0 + n < has[g].x || u0 + n >= has[g].y) continue;
                    const int c = done[g]++, at = place(g, c);
                    if (phase(c) > 0) ok = mbar_wait(&s_empty[at], (phase(c) - 1) & 1, a.err);
                    if (!ok) continue;
                    tc_fence_after();
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int d = 0; d < HD / 16; ++d)
                            tc_mma(tmem + (at * KT + t) * WT_TILE, k + (((g * KT + t) * L::OPER + (d >> 2) * WT_SUB + (d & 3) * 32) >> 4),
                                   q + (((d >> 2) * WT_SUB + (d & 3) * 32) >> 4), id, d != 0);
                    tc_commit(&s_full[at]);
                }
                tc_commit(&q_empty[st]);
            }
            tc_commit(&drain);  // every MMA has ended before TMEM is given back
            mbar_wait(&drain, 0, a.err);
        }
        __syncwarp();
    } else {
        // ---- the sums: a thread has a key of each of its group's key tiles, and its half of the columns ----
        constexpr int COLS = WT_TILE / H, W = COLS / 4, STEPS = 4;  // columns of a warp, of a step
        const int g = warp / (4 * H), h = (warp >> 2) % H, row = tid & (WT_TILE - 1);
        const int2 has = group_range(g);
        const uint32_t lse = smem_addr(sm + L::LSE) + warp * 2 * COLS * 4;
        // the log-sum-exps of the columns of the next tile of rows
        const int heads = a.kv_heads * a.group, first = tokens.x + has.x * per;
        int col_token[COLS / 32];
        const float* from[COLS / 32];
#pragma unroll
        for (int i = 0; i < COLS / 32; ++i) {
            const int c = h * COLS + lane + 32 * i;
            col_token[i] = c / a.group;
            from[i] = a.lse + (long long)(s.row0 + first + col_token[i]) * heads + head * a.group + c - col_token[i] * a.group;
        }
        float l[COLS / 32];  // negated, in log2 units; of columns past the rows -inf: no weight
        auto ask = [&](int u) {
            const int count = min(per, tokens.y - (tokens.x + u * per));
#pragma unroll
            for (int i = 0; i < COLS / 32; ++i) {
                l[i] = INFINITY;
                if (col_token[i] < count) l[i] = *from[i];
                from[i] += per * heads;
            }
        };
        if (has.x < has.y) ask(has.x);
        float sum[KT], lost[KT];  // with compensation
#pragma unroll
        for (int t = 0; t < KT; ++t) sum[t] = lost[t] = 0.f;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + h * COLS;
        bool ok = true;
        for (int u = has.x; u < has.y; ++u) {
            const int c = u - has.x, at = place(g, c);
            const uint32_t lb = lse + (c & 1) * COLS * 4;
#pragma unroll
            for (int i = 0; i < COLS / 32; ++i) asm volatile("st.shared.f32 [%0], %1;" ::"r"(lb + (lane + 32 * i) * 4), "f"(l[i] * -LOG2E) : "memory");
            __syncwarp();
            if (u + 1 < has.y) ask(u + 1);
            const int token = tokens.x + u * per, count = min(per, tokens.y - token), cols = count * a.group;
            // whether every token sees every key of the group's tiles
            const int low = key0 + g * KT * WT_TILE, high = low + KT * WT_TILE - 1, pos = s.base + token;
            const bool full = count == per && pos >= high && (a.window <= 0 || pos + per - 1 < low + a.window);
            ok = wait(&s_full[at], phase(c));
            if (!ok) break;
            tc_fence_after();
            const uint32_t ts = lanes + at * KT * WT_TILE;
            const int steps = full ? STEPS : min(STEPS, (max(0, cols - h * COLS) + W - 1) / W);
            float2 acc[KT][2];
#pragma unroll
            for (int t = 0; t < KT; ++t) acc[t][0] = acc[t][1] = make_float2(0.f, 0.f);
            // (Reading the next columns ahead takes registers, and more time than it saves: 25 prompts of up to 578 tokens 41.6 us, 36.9
            // without, two chunks after 6000 to 9000 keys 567 and 460.)
            float x[KT][W];
            auto read = [&](int i) {
#pragma unroll
                for (int t = 0; t < KT; ++t) tmem_ld_issue<W>(ts + t * WT_TILE + i * W, x[t]);
            };
            auto released = [&]() {  // S is in registers
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&s_empty[at]);
            };
            auto add = [&](int i, auto masked) {  // (a body of its own without masks, which are as much work again)
                int c0[KT], c1[KT];  // columns [c0, c1) of the warp's see the thread's keys
                if (decltype(masked)::value)
#pragma unroll
                    for (int t = 0; t < KT; ++t) {
                        const int ahead = low + t * WT_TILE + row - pos;  // the key's position less the first token's
                        c0[t] = min(max(0, ahead), count) * a.group - h * COLS;
                        c1[t] = (a.window > 0 ? max(0, min(count, ahead + a.window)) : count) * a.group - h * COLS;
                    }
                const float2 scale = make_float2(a.scale_log2, a.scale_log2);
#pragma unroll
                for (int e = 0; e < W / 4; ++e) {
                    float4 z;
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(z.x), "=f"(z.y), "=f"(z.z), "=f"(z.w) : "r"(lb + (i * W + 4 * e) * 4));
#pragma unroll
                    for (int t = 0; t < KT; ++t) {
                        const float* y = x[t] + 4 * e;
                        const float2 v = fma2(make_float2(y[0], y[1]), scale, make_float2(z.x, z.y));
                        const float2 w = fma2(make_float2(y[2], y[3]), scale, make_float2(z.z, z.w));
                        float2 p = make_float2(ex2(v.x), ex2(v.y)), q = make_float2(ex2(w.x), ex2(w.y));
                        if (decltype(masked)::value) {
                            const int at = i * W + 4 * e;
                            p.x = at >= c0[t] && at < c1[t] ? p.x : 0.f;
                            p.y = at + 1 >= c0[t] && at + 1 < c1[t] ? p.y : 0.f;
                            q.x = at + 2 >= c0[t] && at + 2 < c1[t] ? q.x : 0.f;
                            q.y = at + 3 >= c0[t] && at + 3 < c1[t] ? q.y : 0.f;
                        }
                        acc[t][0] = add2(acc[t][0], p);
                        acc[t][1] = add2(acc[t][1], q);
                    }
                }
            };
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                if (i >= steps) break;
                read(i);
                tmem_ld_wait();
#pragma unroll
                for (int t = 0; t < KT; ++t) tmem_ld_done(x[t]);
                if (i + 1 == steps) released();
                if (full)
                    add(i, std::false_type());
                else
                    add(i, std::true_type());
            }
            if (steps == 0) released();
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                const float y = ((acc[t][0].x + acc[t][0].y) + (acc[t][1].x + acc[t][1].y)) - lost[t], v = sum[t] + y;
                lost[t] = (v - sum[t]) - y;
                sum[t] = v;
            }
        }
        if constexpr (H == 2) {  // the halves' sums as one
            float* other = reinterpret_cast<float*>(sm + L::LSE) + (warp & ~7) * 2 * COLS + row;  // (the group's log-sum-exps are done with)
            asm volatile("bar.sync %0, 256;" ::"r"(1 + g) : "memory");
            if (h == 1)
#pragma unroll
                for (int t = 0; t < KT; ++t) other[t * WT_TILE] = sum[t];
            asm volatile("bar.sync %0, 256;" ::"r"(1 + g) : "memory");
            if (h == 0)
#pragma unroll
                for (int t = 0; t < KT; ++t) sum[t] += other[t * WT_TILE];
        }
        if (ok && h == 0)
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                const int key = key0 + (g * KT + t) * WT_TILE + row;
                if (key >= key1 || key < lowest) continue;
                if (a.segments > 1) {
                    part[key - key0] = sum[t];
                } else {
                    float* out = a.weights + slot * a.w_slot + (long long)head * a.width + key;
                    *out = key < s.base ? *out + sum[t] : sum[t];
                }
            }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == L::MMA) tmem_dealloc(tmem, L::TM_COLS);
}

template <class T, int HD, int TILES>
cudaError_t launch_tiles(const WeightsArgs& a, const CUtensorMap& map, const CUtensorMap& q_map, bool q_tma, int key_tiles, cudaStream_t s) {
    using L = WtLayout<HD, TILES>;
    const auto kern = key_weights_tc_kernel<T, HD, TILES>;
    const cudaError_t e = ensure_kernel_smem(reinterpret_cast<const void*>(kern), L::BYTES);
    if (e != cudaSuccess) return e;
    return launch_ex(kern, dim3((key_tiles + TILES - 1) / TILES * a.kv_heads, a.slots, a.segments), L::THREADS, L::BYTES, s, 1, a, map, q_map, (int)q_tma);
}
template <class T, int HD>
cudaError_t launch_tc(const WeightsArgs& a, const CUtensorMap& map, const CUtensorMap& q_map, bool q_tma, int key_tiles, cudaStream_t s) {
    return a.tiles == 1 ? launch_tiles<T, HD, 1>(a, map, q_map, q_tma, key_tiles, s) : launch_tiles<T, HD, 4>(a, map, q_map, q_tma, key_tiles, s);
}

}  // namespace

cudaError_t launch_weights_tc(const WeightsArgs& a, const CUtensorMap& map, const CUtensorMap& q_map, bool q_tma, int dtype,
                              int key_tiles, cudaStream_t s) {
    if (dtype == MTP_BF16)
        return a.dim == 64 ? launch_tc<Bf16, 64>(a, map, q_map, q_tma, key_tiles, s) : launch_tc<Bf16, 128>(a, map, q_map, q_tma, key_tiles, s);
    return a.dim == 64 ? launch_tc<F16, 64>(a, map, q_map, q_tma, key_tiles, s) : launch_tc<F16, 128>(a, map, q_map, q_tma, key_tiles, s);
}

}  // namespace mtp
