// chunk_attention_tc.cu -- the kernel of mtp_chunk_attention for more than 16 rows per slot
// and key head (prompts, chunks): tcgen05, shares of the unit stream (chunk.cuh) of 128 or
// 256 packed rows by 128 keys.
//
//   S = Q K^T          128 x 64 fp32 in TMEM per tile of 128 rows and step of 64 keys
//   P = 2^(c S - m)    a row per thread, written over S as 16-bit values (c = scale log2 e)
//   O += P V           P read from TMEM, V as an MN-major operand, 128 x head_dim fp32 in TMEM
//
// A tile has four softmax warps and two places for S: while a step's scores are in the hands of
// the softmax, the tensor cores make the next step's, so that the softmax warps go from step
// to step without waiting.  (With one place of 128 keys softmax and MMAs took turns: 4500
// cycles per 128 keys of two tiles, of which the MMAs fill 2048.  The price of N = 64 is its
// Q, read per 64 keys: 45 cycles per MMA where 32 would do.)  An SM has two tiles: those of one
// CTA, which take turns at the tensor cores (128 dims), or two CTAs' (64 dims).
// A tile's MMAs are issued by a thread of its own: one for both spent more time on its waits
// and branches (126 cycles for a barrier that is complete) than the MMAs took.  The issuing
// threads run over the items of the share without a stop, as do the rings of keys and of
// values, which a warp each fills with TMA copies, a lane per page piece; the values' warp brings
// Q too, by a tensor map, where the heads of a key head divide 128 and rows are aligned to 16 bytes
// (25 prompts 41.6 us; brought by the softmax warps, as other rows are, 44.7).  A tile skips the
// steps of which its rows see no key.
//
// Two chunks of 2000 to 4000 tokens after 6000 to 9000, 32 heads on 8 of 128 dims (648 GFLOP): 446 to 471 us
// (GPUs differ), 1380 to 1450 TFLOP/s, of the measured peak (cuBLAS, 1922) about three quarters; the MMAs of 45 and 64
// cycles fill about as much of the time.  64 dims, 16 heads (162 GFLOP): 212 us, 764 TFLOP/s: bound by
// the softmax, whose 64 exponentials a row and step are as many as with 128 dims; a warp issues in
// 44 % of the cycles and waits for results of its own the most.  25 prompts of 182 to 578 tokens,
// 16 heads of 64: 41.6 us, of which the plan is 4, and items of 1 to 5 units with a start and
// end each the rest.
//
// Code size matters: with everything unrolled and inlined (190 KB) the warps waited for
// instructions, 10,000 cycles per 128 keys.
//
// m is a row's reference, not its maximum: the weights are made with the one that is there, and
// only where a step's weights add up to more than 2^15 (or a row has none yet) is the maximum
// looked for, the reference moved and the output in TMEM rescaled.  After a row's first steps
// that is rare, and 64 maxima per row and step are saved.  bf16 weights have the same relative
// precision whatever the reference is; fp16 ones too, down to 2^-14 of the reference's weight, below it
// they are multiples of 2^-24 of it.  The sum takes the weights before they are rounded, in fp32.
// P is rounded once to the type: a second product with its residues would cost half as much
// tensor time again, and the error (as large as the output's own rounding to 16 bits) is
// within the type.  Q, K and V enter as they are.
// RES: up to 32 rows, where memory leaves the tensor cores time, P enters with its residues,
// which go to the other half of S's place and have a product of their own.  (8 slots of 4,000
// to 30,000 keys, 32 rows each, 128 dims fp16: 93.6 us, 86.9 without; 32 slots of up to 2000 keys,
// 64 dims bf16: 22.3 and 19.1.)
#include <algorithm>
#include <climits>
#include <type_traits>

#include "chunk.cuh"
#include "tcgen05.cuh"

namespace mtp {
namespace {

constexpr int CT_TILE = 128, CT_KEYS = 128;
constexpr int CT_STEP = CH_STEP;        // keys of a step: the scores that a thread holds
constexpr uint32_t CT_SUB = 128 * 128;  // 128 rows of 128 bytes
constexpr int CT_HANDOVER = 2;  // MMAs of S before whose end the other tile may go on
constexpr float LAG = 8.f, LIMIT = 32768.f;
constexpr float LN2 = 0.69314718055994531f;

// Tiles, warps and shared memory of a CTA.
template <int HD>
struct CtLayout {
    static constexpr int TILES = chunk_tc_tiles(HD), STAGES = 4;  // stages: of K and of V, 64 keys each
    static constexpr int MMA = 4 * TILES, COPY_K = 5 * TILES, COPY_V = COPY_K + 1;  // the first MMA warp, the copying warps
    static constexpr int WARPS = (COPY_V + 4) / 4 * 4, THREADS = WARPS * 32;
    // TMEM: tile t, step s: S at 128 t + 64 (s & 1), O after the tiles' S
    static constexpr uint32_t TM_S = 0, TM_O = 128 * TILES, TM_O_TILE = 128, TM_COLS = TILES == 1 ? 256 : 512;
    static constexpr uint32_t OPER = CT_SUB * (HD / 64);  // a tile of Q
    static constexpr uint32_t ATOM = CT_STEP * 128, STEP = ATOM * (HD / 64);  // 64 columns of a stage; a stage
    static constexpr uint32_t K = TILES * OPER, V = K + STAGES * STEP, OUT = V + STAGES * STEP;  // OUT: 64 columns of a tile's rows
    static constexpr size_t BYTES = 1024 + OUT + TILES * CT_SUB;
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
__device__ __forceinline__ void tma_cache(void* dst, const CUtensorMap* map, int x, int row, int block, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            smem_addr(dst)),
        "l"(map), "r"(x), "r"(row), "r"(block), "r"(smem_addr(bar))
        : "memory");
}
// Whether a barrier's phase is complete, without waiting (try_wait suspends the thread for a while where it is not).
__device__ __forceinline__ bool mbar_test(uint64_t* bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_addr(bar)), "r"(parity)
        : "memory");
    return done != 0;
}
// One thread of the (whole) warp, the same at every call.
__device__ __forceinline__ bool elect_one() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}
// D = A B (+ D), A (16-bit, K-major) in TMEM: lane = row, two K elements per column
__device__ __forceinline__ void tc_mma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(acc)
        : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
        "%15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// V's 128-byte-swizzled rows as an MN-major operand: 64-column atoms `atom` bytes apart
__device__ __forceinline__ uint64_t v_desc(uint32_t saddr, uint32_t atom) {
    uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(atom >> 4) << 16;    // between 64-column atoms
    d |= (uint64_t)(1024 >> 4) << 32;    // between groups of 8 keys
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
template <class T>
constexpr uint32_t ct_idesc(int n, bool b_mn) {  // f16_idesc's types are bf16; fp16's codes are 0
    return std::is_same<T, Bf16>::value ? f16_idesc(CT_TILE, n, b_mn) : f16_idesc(CT_TILE, n, b_mn) & ~((1u << 7) | (1u << 10));
}

// What a tile (0 or 1) of an item does in this CTA: its rows, and the steps [from, to) of the
// item (two to a unit), of the share's, of which its rows see a key.
struct CtTile {
    int p0, rows, from, to;
    __device__ __forceinline__ CtTile(const ChunkWalk& w, int tile) {
        p0 = w.t.p0 + tile * CT_TILE;
        rows = max(0, min(CT_TILE, w.t.rows - tile * CT_TILE));
        from = max(2 * w.k0, tile ? w.t.steps.z : w.t.steps.x);
        to = max(from, min(2 * w.k1, tile ? w.t.steps.w : w.t.steps.y));
    }
};

template <class T, int HD, bool RES>
__global__ void __launch_bounds__(CtLayout<HD>::THREADS, 3 - CtLayout<HD>::TILES) chunk_tc_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap q_map) {
    using L = CtLayout<HD>;
    constexpr int ST = L::STAGES, TILES = L::TILES;
    constexpr uint32_t TM_S = L::TM_S, TM_O = L::TM_O;
    extern __shared__ unsigned char ct_raw[];
    __shared__ uint64_t q_full[TILES], q_empty[TILES], s_full[TILES][2], p_full[TILES][2], pv_done[TILES][2], k_full[ST], k_empty[ST], v_full[ST], v_empty[ST], turn[TILES], drain[TILES];
    __shared__ uint32_t tmem_base;
    unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(ct_raw) + 1023) & ~(uintptr_t)1023);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    if (warp == L::MMA) {
        tmem_alloc(&tmem_base, L::TM_COLS);
        tmem_relinquish();
    }
    if (tid == 0) {
        for (int i = 0; i < TILES; ++i) {
            mbar_init(&drain[i], 1);
            mbar_init(&turn[i], 1);
            mbar_init(&q_full[i], a.q_tma ? 1 : 4);
            mbar_init(&q_empty[i], 1);
            for (int h = 0; h < 2; ++h) {
                mbar_init(&s_full[i][h], 1);
                mbar_init(&p_full[i][h], 4);
                mbar_init(&pv_done[i][h], 1);
            }
        }
        for (int i = 0; i < ST; ++i) {
            mbar_init(&k_full[i], 1);
            mbar_init(&k_empty[i], TILES);  // every tile's MMAs
            mbar_init(&v_full[i], 1);
            mbar_init(&v_empty[i], TILES);
        }
        fence_barrier_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    pdl_launch_dependents();
    pdl_wait();  // the plan
    const ChunkStart start = a.start[cta];
    const int units = start.units;
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        return __all_sync(FULL_MASK, mbar_try_wait(bar, parity & 1) || chunk_wait(bar, parity, a.err)) != 0;
    };

    if (units > 0) {
        if (warp == L::COPY_K || warp == L::COPY_V) {
            // ---- copies of the keys or the values: a lane per piece of a step ----
            const int kv = warp == L::COPY_V, P = 1 << a.page_shift, box = min(P, CT_STEP), per = CT_STEP / box;
            const int sub = lane % per, half = lane / per;
            const bool mine = half < HD / 64;
            unsigned char* ring = sm + (kv ? L::V : L::K) + half * L::ATOM + sub * box * 128;
            uint64_t *full = kv ? v_full : k_full, *empty = kv ? v_empty : k_empty;
            ChunkWalk w(start);
            int step = 2 * w.k0, n = 0;
            bool ok = true;
            // pages [base, base + 32) of the slot, one per lane, and the 32 after them
            int base = 0, pages = 0, ahead = 0, key_first = 0, hi = 0, lo = 0, last = 0, head_block = 0;
            const int* table = nullptr;
            auto lookup = [&](int first) { return first + lane < a.bt_stride ? *(table + first + lane) : -1; };
            int queries[TILES] = {};  // tiles of Q copied so far
            auto enter = [&]() {  // an item's first step
                if (kv && a.q_tma)  // the values' warp, which is behind the keys', copies Q too
#pragma unroll
                    for (int tile = 0; tile < TILES; ++tile) {
                        const CtTile x(w, tile);
                        if (x.from >= x.to) continue;
                        if (queries[tile] > 0) ok = ok && wait(&q_empty[tile], queries[tile] - 1);
                        ++queries[tile];
                        if (ok && lane == 0) {
                            mbar_arrive_expect_tx(&q_full[tile], L::OPER);
                            for (int h = 0; h < HD / 64; ++h)
                                tma_cache(sm + tile * L::OPER + h * CT_SUB, &q_map, h * 64, w.head * a.group,
                                          w.t.row0 + chunk_token(a, x.p0), &q_full[tile]);
                        }
                    }
                table = a.block_table + (size_t)w.t.slot * a.bt_stride;
                key_first = w.key0<CT_KEYS>();
                hi = w.t.hi;
                lo = w.t.lo;
                last = 2 * w.k1;
                head_block = a.layer_block + kv * a.kv_heads + w.head;
                base = (key_first + step * CT_STEP) >> a.page_shift & ~31;
                pages = lookup(base);
                ahead = lookup(base + 32);
            };
            enter();
            for (const int steps = 2 * units; ok && n < steps; ++n) {
                const int st = n % ST, key = key_first + step * CT_STEP + sub * box, index = key >> a.page_shift;
                if (index - base >= 32) {  // (the same in all lanes: a step's pages lie in one aligned group)
                    base += 32;
                    pages = ahead;
                    ahead = lookup(base + 32);
                }
                int page = __shfl_sync(FULL_MASK, pages, (index - base) & 31);
                page = page >= 0 && page < a.n_pages ? page : -1;  // -1: outside the pool, zeros
                const int block = page < 0 ? -1 : page * a.page_blocks + head_block;
                const bool wanted = mine && key < hi && key + box > lo;  // some row sees a key of the piece
                const uint32_t bytes = __popc(__ballot_sync(FULL_MASK, wanted)) * box * 128;
                if (n >= ST && !(ok = wait(&empty[st], n / ST - 1))) break;
                if (lane == 0) mbar_arrive_expect_tx(&full[st], bytes);
                __syncwarp();
                if (wanted) tma_cache(ring + st * L::STEP, &map, half * 64, key & (P - 1), block, &full[st]);
                if (++step == last && n + 1 < steps) {
                    w.next(a);
                    step = 0;
                    enter();
                }
            }
            if (!ok && lane == 0)  // what is in flight lands before the CTA leaves
                for (int i = max(0, n - ST); i < n; ++i) chunk_wait(&full[i % ST], i / ST, nullptr);
            if (!ok && lane == 0 && kv && a.q_tma)
                for (int tile = 0; tile < TILES; ++tile)
                    if (queries[tile] > 0) chunk_wait(&q_full[tile], queries[tile] - 1, nullptr);
            __syncwarp();
        } else if (warp >= L::MMA && warp < L::MMA + TILES) {
            // ---- MMAs of a tile, by one thread ----
            if (elect_one()) {
                constexpr uint32_t IDESC_S = ct_idesc<T>(CT_STEP, false), IDESC_O = ct_idesc<T>(HD, true);
                const int tile = warp - L::MMA;
                ChunkWalk w(start);
                CtTile x(w, tile), y = x;  // y: the unit before's
                const uint64_t q = sw128_desc(smem_addr(sm + tile * L::OPER)), k0 = sw128_desc(smem_addr(sm + L::K)),
                               v0 = v_desc(smem_addr(sm + L::V), L::ATOM);
                const uint32_t s_tmem = tmem + TM_S + tile * 128, o_tmem = tmem + TM_O + tile * L::TM_O_TILE;
                uint32_t q_phase = 0, p_phase[2] = {0, 0};
                bool ok = true;
                auto await = [&](bool there, uint64_t* bar, uint32_t phase) { ok = ok && (there || chunk_wait(bar, phase, a.err)); };
                int k = w.k0, k1 = w.k1;
                // the products of the steps of unit n - 1, between them the scores of unit n's: S of a step comes after
                // the P V of two steps before, in whose place it goes, and the softmax has the step between to work on
                for (int n = 0; ok && n <= units; ++n) {
                    const int at = k - 1;
                    const bool more = n < units;
                    if (n > 0 && k == k1) {
                        w.next(a);
                        k = 0;
                        k1 = w.k1;
                        x = CtTile(w, tile);
                    }
                    // S of a step, whose keys are there; `hand`: the turn goes to the other tile under it
                    auto scores = [&](int half, int st, bool hand) {
                        const int step = 2 * k + half;
                        if (step >= x.from && step < x.to) {  // S = Q K^T
                            if (step == x.from) {
                                await(false, &q_full[tile], q_phase++);
                                if (!ok) return;
                                tc_fence_after();
                            }
                            const uint64_t kd = k0 + st * (L::STEP >> 4);
#pragma unroll
                            for (int d = 0; d < HD / 16; ++d) {
                                if (hand && d == HD / 16 - CT_HANDOVER) mbar_arrive(&turn[tile ^ 1]);  // (seen by the time that S is through)
                                tc_mma(s_tmem + half * 64, q + (((d >> 2) * CT_SUB + (d & 3) * 32) >> 4),
                                       kd + (((d >> 2) * L::ATOM + (d & 3) * 32) >> 4), IDESC_S, d != 0);
                            }
                            tc_commit(&s_full[tile][half]);
                            if (step + 1 == x.to) tc_commit(&q_empty[tile]);
                        } else if (hand) {
                            mbar_arrive(&turn[tile ^ 1]);
                        }
                        tc_commit(&k_empty[st]);
                    };
                    // at an item's first unit both products come first: its Q may still be on its way, and the item before
                    // waits for its last product
                    const bool entering = n > 0 && k == 0;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int i = 2 * n + half, st = i % ST, before = (i + ST - 2) % ST;
                        const int p_step = 2 * at + half;
                        const bool p_on = n > 0 && p_step >= y.from && p_step < y.to;
                        // all barriers are asked at once: an answer takes 126 cycles
                        const bool k_there = !more || mbar_try_wait(&k_full[st], (i / ST) & 1);
                        const bool v_there = n == 0 || mbar_try_wait(&v_full[before], ((i - 2) / ST) & 1);
                        const bool p_there = !p_on || mbar_try_wait(&p_full[tile][half], p_phase[half] & 1);
                        // The tiles take turns, so that a tile's MMAs run in one piece and their results come half a step apart:
                        // mixed, both tiles' scores would be ready late, and both softmax groups wait for them.
                        const bool my_turn = TILES == 1 || (tile == 0 && i == 0);
                        const uint32_t turn_phase = i - 1 + tile;
                        const bool turn_there = my_turn || mbar_try_wait(&turn[tile], turn_phase & 1);
                        await(k_there, &k_full[st], i / ST);
                        await(v_there, &v_full[before], (i - 2) / ST);
                        await(p_there, &p_full[tile][half], p_phase[half]);
                        await(turn_there, &turn[tile], turn_phase);
                        if (!ok) break;
                        tc_fence_after();
                        if (p_on) {  // O += P V
                            p_phase[half]++;
                            const uint64_t v = v0 + before * (L::STEP >> 4);
#pragma unroll
                            for (int d = 0; d < CT_STEP / 16; ++d)
                                tc_mma_ta(o_tmem, s_tmem + half * 64 + d * 8, v + d * (2048 >> 4), IDESC_O, d != 0 || p_step != y.from);
                            if constexpr (RES)
#pragma unroll
                                for (int d = 0; d < CT_STEP / 16; ++d)
                                    tc_mma_ta(o_tmem, s_tmem + half * 64 + 32 + d * 8, v + d * (2048 >> 4), IDESC_O, 1);
                            tc_commit(&pv_done[tile][half]);
                        }
                        if (n > 0) tc_commit(&v_empty[before]);
                        if (more && !entering)
                            scores(half, st, TILES == 2);
                        else if (TILES == 2)
                            mbar_arrive(&turn[tile ^ 1]);
                    }
                    if (ok && more && entering)
#pragma unroll 1
                        for (int half = 0; half < 2; ++half) scores(half, (2 * n + half) % ST, false);
                    y = x;
                    ++k;
                }
                tc_commit(&drain[tile]);  // every MMA has ended before TMEM is given back
                chunk_wait(&drain[tile], 0, a.err);
            }
            __syncwarp();
        } else if (warp < 4 * TILES) {
            // ---- softmax: group g has tile g, a row per thread ----
            const int g = warp >> 2, r = tid & 127;
            const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), ts = lanes + TM_S + g * 128, to = lanes + TM_O + g * L::TM_O_TILE;
            unsigned char* qs = sm + g * L::OPER;
            const int heads = a.kv_heads * a.group;
            ChunkWalk w(start);
            CtTile x(w, g);
            int n = 0, seen[2] = {0, 0};  // steps of either half, which s_full and pv_done count too
            bool ok = true;
            // a row's place in q and out, without the strides
            auto place = [&](const ChunkWalk& w, int p, int& head) {
                const int token = chunk_token(a, p);
                head = w.head * a.group + p - token * a.group;
                return (long long)w.t.row0 + token;
            };
            // Q of an item on its way into shared memory: a warp brings its own 32 rows, 16 bytes a thread and step,
            // HD / 8 threads to a row; rows past the tile are zeros
            auto load_q = [&](const ChunkWalk& w, const CtTile& x) {
                constexpr int PER = HD / 8, ROWS = 32 / PER;
                int head;
                const long long row = place(w, x.p0 + min(r, max(x.rows - 1, 0)), head);
                const long long mine = row * a.q_stride + head * HD;
                const int c = lane % PER;
#pragma unroll 4
                for (int i = 0; i < 32; i += ROWS) {
                    const int from = i + lane / PER, at = (r & ~31) + from;
                    const uint16_t* src = a.q + __shfl_sync(FULL_MASK, mine, from) + c * 8;
                    unsigned char* dst = qs + (c >> 3) * CT_SUB + at * 128 + (((c & 7) ^ (at & 7)) << 4);
                    const bool live = at < x.rows;
                    if (a.q_vec) {
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(dst)), "l"(src), "r"(live ? 16 : 0) : "memory");
                    } else {
                        uint32_t v[4] = {0u, 0u, 0u, 0u};
                        if (live)
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = (uint32_t)*(src + 2 * e) | (uint32_t)*(src + 2 * e + 1) << 16;
                        *reinterpret_cast<uint4*>(dst) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                }
            };
            auto q_there = [&]() {
                asm volatile("cp.async.wait_all;" ::: "memory");
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(&q_full[g]);
            };
            const bool bring_q = !a.q_tma;  // rows that a tensor map cannot describe
            if (bring_q && x.from < x.to) {
                load_q(w, x);
                q_there();
            }
            for (;;) {
                const int len = w.k1 - w.k0;
                // (rows past the tile's are not looked at: as if they saw every key)
                const int pos = r < x.rows ? w.t.base + chunk_token(a, x.p0 + r) : INT_MAX;
                const int window = a.window > 0 && r < x.rows ? a.window : INT_MAX;
                // steps [inner_from, inner_to): every row of the warp sees all of their keys (and some row of the item does,
                // where the warp has none)
                const int key_first = w.key0<CT_KEYS>(), hi = w.t.hi, lo = w.t.lo, share = 2 * (n - w.k0);
                const int pos0 = __reduce_min_sync(FULL_MASK, pos), pos1 = __reduce_max_sync(FULL_MASK, r < x.rows ? pos : INT_MIN);
                int inner_to = (hi - key_first) / CT_STEP, inner_from = (lo - key_first + CT_STEP - 1) / CT_STEP;
                if (pos0 < hi) inner_to = pos0 < key_first ? 0 : min(inner_to, (pos0 + 1 - key_first) / CT_STEP);
                if (a.window > 0 && pos1 >= a.window + key_first) inner_from = max(inner_from, (pos1 - a.window - key_first) / CT_STEP + 1);
                const bool own = r < x.rows;  // (what stands in Q's other rows, NaN perhaps, is no reason to look for a reference)
                float ref = own ? -INFINITY : 0.f, sum = 0.f;
                bool asked = false;  // Q of the item after this one is on its way
                auto ask_q = [&]() {
                    ChunkWalk next = w;
                    next.next(a);
                    if (next.left <= 0) return;
                    const CtTile y(next, g);
                    asked = y.from < y.to;
                    if (asked) load_q(next, y);
                };
                bool there = false;  // the step's scores are known to be there
                float s0[32], s1[32];
#pragma unroll 1
                for (int step = x.from; step < x.to; ++step) {
                    const int half = step & 1;
                    const uint32_t tsh = ts + half * 64;
                    const bool inner = step >= inner_from && step < inner_to, onward = step + 1 < x.to;
                    ok = __all_sync(FULL_MASK, there || chunk_wait(&s_full[g][half], half ? seen[1] : seen[0], a.err)) != 0;
                    if (!ok) break;
                    tc_fence_after();
                    tmem_ld_issue<32>(tsh, s0);
                    tmem_ld_issue<32>(tsh + 32, s1);
                    if (half) ++seen[1]; else ++seen[0];
                    const uint32_t next_phase = half ? seen[0] : seen[1];
                    if (!onward && bring_q) ask_q();  // the tile's last S is there: Q's space is free
                    __syncwarp();
                    tmem_ld_wait();
                    tmem_ld_done(s0);
                    tmem_ld_done(s1);
                    if (!inner) {
                        // columns (lowest, highest] of the step are the keys that this row sees
                        const int key0 = key_first + step * CT_STEP, highest = pos - key0, lowest = pos - key0 >= window ? pos - key0 - window : -1;
                        auto below = [](int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; };  // columns [0, n)
                        const unsigned long long sees = below(highest + 1) & ~below(lowest + 1);
                        const uint32_t m0 = (uint32_t)sees, m1 = (uint32_t)(sees >> 32);
#pragma unroll
                        for (int c = 0; c < 32; ++c) {
                            s0[c] = m0 >> c & 1 ? s0[c] : -INFINITY;
                            s1[c] = m1 >> c & 1 ? s1[c] : -INFINITY;
                        }
                    }
                    float2 acc[2];
                    auto weights32 = [&](const float (&x)[32], uint32_t at) {  // over S, which is all in registers
                        constexpr int N = RES ? 8 : 16;  // weights in registers, in pairs
#pragma unroll
                        for (int e0 = 0; e0 < 16; e0 += N) {
                            uint32_t y[N], rest[N];
#pragma unroll
                            for (int e = 0; e < N; ++e) {
                                const float2 z = fma2(make_float2(x[2 * (e0 + e)], x[2 * (e0 + e) + 1]),
                                                      make_float2(a.scale_log2, a.scale_log2), make_float2(-ref, -ref));
                                const float2 p = make_float2(ex2(z.x), ex2(z.y));
                                acc[e & 1] = add2(acc[e & 1], p);
                                y[e] = T::pack(p.x, p.y);
                                if (RES) rest[e] = T::pack(p.x - T::to_float((uint16_t)y[e]), p.y - T::to_float((uint16_t)(y[e] >> 16)));
                            }
                            tmem_st(at + e0, y);
                            if (RES) tmem_st(at + 32 + e0, rest);
                        }
                    };
                    auto weights = [&]() {  // their sum
                        acc[0] = acc[1] = make_float2(0.f, 0.f);
                        weights32(s0, tsh);
                        weights32(s1, tsh + 16);
                        return (acc[0].x + acc[0].y) + (acc[1].x + acc[1].y);
                    };
                    float part = 0.f;
                    bool fits = __all_sync(FULL_MASK, ref != -INFINITY);  // every row has a reference
                    if (fits) {
                        part = weights();
                        fits = __all_sync(FULL_MASK, part <= LIMIT || !own);
                    }
                    if (!fits) {
                        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                        for (int c = 0; c < 32; c += 2) {
                            mx[0] = fmaxf(mx[0], s0[c]);
                            mx[1] = fmaxf(mx[1], s0[c + 1]);
                            mx[2] = fmaxf(mx[2], s1[c]);
                            mx[3] = fmaxf(mx[3], s1[c + 1]);
                        }
                        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale_log2;
                        const bool moves = top > ref + LAG;  // (from -inf: any value)
                        const float f = moves ? ex2(ref - top) : 1.f;
                        if (moves) ref = top;
                        sum *= f;
                        __syncwarp();
                        if (step > x.from) {  // the product before is complete, the next one waits for this step's weights
                            ok = wait(&pv_done[g][half ^ 1], next_phase - 1);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < HD; c += 16) {
                                float v[16];
                                tmem_ld<16>(to + c, v);
                                uint32_t y[16];
#pragma unroll
                                for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(v[e] * f);
                                tmem_st(to + c, y);
                            }
                        }
                        const float kept = ref;
                        if (ref == -INFINITY) ref = 0.f;  // a row that has seen no key: every weight 0
                        part = weights();
                        ref = kept;
                    }
                    sum += part;
                    there = onward && mbar_test(&s_full[g][half ^ 1], next_phase & 1);  // (the answer is there when it is needed)
                    if (!inner) {
                        // keys of the step that no row of the item sees: whatever their values are, zeros in their place (both
                        // groups write them, each before its own product)
                        const int key0 = key_first + step * CT_STEP;
                        if (key0 + CT_STEP > hi || key0 < lo) {
                            const int i = share + step;  // of the share's steps
                            ok = wait(&v_full[i % ST], i / ST);
                            if (!ok) break;
                            const int row = r & (CT_STEP - 1), key = key0 + row;
                            if (key >= hi || key < lo) {
                                unsigned char* v = sm + L::V + (uint32_t)(i % ST) * L::STEP + row * 128;
                                for (int c = r / CT_STEP; c < HD / 8; c += 128 / CT_STEP)
                                    *reinterpret_cast<uint4*>(v + (c >> 3) * L::ATOM + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                            }
                            fence_proxy_async();
                        }
                    }
                    __syncwarp();
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[g][half]);
                }
                if (!ok) break;
                if (bring_q) {
                    if (x.from >= x.to) ask_q();  // (nothing here: Q's space was free already)
                    if (asked) q_there();
                }
                // ---- the item's rows ----
                const bool any = x.from < x.to;
                if (any) {
                    const int half = (x.to - 1) & 1;
                    ok = wait(&pv_done[g][half], (half ? seen[1] : seen[0]) - 1);
                    if (!ok) break;
                    tc_fence_after();
                }
                const bool begins = w.begins(), whole = begins && w.ends();
                int head;
                const long long row = place(w, x.p0 + r, head);
                const bool live = r < x.rows;
                const float f = sum == 0.f ? 0.f : 1.f / sum;  // (no key: 0)
                const long long mine = row * a.out_stride + head * HD;
                float* part = a.part + ((size_t)cta * 2 + begins) * (CT_TILE * TILES) * (HD + 2);
#pragma unroll 1
                for (int c = 0; c < HD; c += 64) {
                    float v[2][32];
                    __syncwarp();
                    if (any) {
                        tmem_ld_issue<32>(to + c, v[0]);
                        tmem_ld_issue<32>(to + c + 32, v[1]);
                        tmem_ld_wait();
                        tmem_ld_done(v[0]);
                        tmem_ld_done(v[1]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[0][e] = v[1][e] = 0.f;
                    }
                    if (whole) {
                        // through shared memory, a warp its own 32 rows: eight threads write a row's 128 bytes
                        unsigned char* stage = sm + L::OUT + g * CT_SUB;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float* z = v[e >> 2] + (e & 3) * 8;
                            uint4 y;
                            y.x = T::pack(z[0] * f, z[1] * f);
                            y.y = T::pack(z[2] * f, z[3] * f);
                            y.z = T::pack(z[4] * f, z[5] * f);
                            y.w = T::pack(z[6] * f, z[7] * f);
                            *reinterpret_cast<uint4*>(stage + r * 128 + ((e ^ (r & 7)) << 4)) = y;
                        }
                        __syncwarp();
#pragma unroll 4
                        for (int i = 0; i < 32; i += 4) {
                            const int from = i + (lane >> 3), at = (r & ~31) + from;
                            uint16_t* dst = a.out + __shfl_sync(FULL_MASK, mine, from) + c + (lane & 7) * 8;
                            const uint4 y = *reinterpret_cast<const uint4*>(stage + at * 128 + (((lane & 7) ^ (at & 7)) << 4));
                            if (at >= x.rows) continue;
                            if (a.out_vec) {
                                *reinterpret_cast<uint4*>(dst) = y;
                            } else {
                                const uint32_t z[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    dst[2 * e] = (uint16_t)z[e];
                                    dst[2 * e + 1] = (uint16_t)(z[e] >> 16);
                                }
                            }
                        }
                    } else if (live) {
                        float4* dst = reinterpret_cast<float4*>(part + (g * CT_TILE + r) * HD + c);
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float* z = v[e >> 3] + (e & 7) * 4;
                            dst[e] = make_float4(z[0], z[1], z[2], z[3]);
                        }
                    }
                }
                if (live && whole && a.lse) a.lse[row * heads + head] = sum == 0.f ? -INFINITY : LN2 * (ref + log2f(sum));
                if (live && !whole) *reinterpret_cast<float2*>(part + (CT_TILE * TILES) * HD + 2 * (g * CT_TILE + r)) = make_float2(ref, sum);
                tc_fence_before();  // O is read before the next item's product overwrites it
                n += len;
                w.next(a);
                if (w.left <= 0) break;
                x = CtTile(w, g);
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    if (warp == L::MMA) tmem_dealloc(tmem, L::TM_COLS);
}

template <class T, int HD, bool RES>
cudaError_t launch_tc(const ChunkArgs& a, const CUtensorMap& map, const CUtensorMap& q_map, cudaStream_t s) {
    const auto kern = chunk_tc_kernel<T, HD, RES>;
    const cudaError_t e = ensure_kernel_smem(reinterpret_cast<const void*>(kern), CtLayout<HD>::BYTES);
    return e == cudaSuccess ? launch_ex(kern, dim3(a.ctas), CtLayout<HD>::THREADS, CtLayout<HD>::BYTES, s, 1, a, map, q_map) : e;
}

}  // namespace

cudaError_t launch_chunk_tc(const ChunkArgs& a, const CUtensorMap& map, const CUtensorMap& q_map, int head_dim, int dtype,
                            cudaStream_t s) {
    auto launch = [&](auto type, auto res) {
        using T = decltype(type);
        constexpr bool RES = decltype(res)::value;
        return head_dim == 64 ? launch_tc<T, 64, RES>(a, map, q_map, s) : launch_tc<T, 128, RES>(a, map, q_map, s);
    };
    if (dtype == MTP_BF16) return a.residues ? launch(Bf16{}, std::true_type{}) : launch(Bf16{}, std::false_type{});
    return a.residues ? launch(F16{}, std::true_type{}) : launch(F16{}, std::false_type{});
}

}  // namespace mtp
