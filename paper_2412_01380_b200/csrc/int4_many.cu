// Products of groups of many rows with 4-bit weights on the fifth-generation tensor cores: y[r] = W[e(r)] rows[r], and
// h[r] = silu(Wg[e(r)] rows[r]) * (Wu[e(r)] rows[r]), W[o][i] = (code - 8) * S[i / 128][o].
//
// A scale belongs to an output and 128 inputs, so it stays out of the MMAs: these multiply (code - 8) / 64, which bfloat16 holds exactly,
// by the rows as they are, and each group's sums are added, times 64 times the scale, to binary32 sums in registers.
// A block's tile is 256 outputs (gate/up: the 128 gate and the 128 up rows of the same outputs) by up to 128 rows.  The weights are
// the M side, in two halves of 128, and the rows the N side, as many columns as there are rows (in sixteens), so that:
//   * a thread that takes sums out has one output: one scale per half and group, and gate and up of its output;
//   * the weights, which have to pass through registers anyway, go from there to tensor memory and never to shared memory, where the
//     rows need the room to be read twice, once per half (128 columns by 256 outputs: 32 + 16 KB in and 64 + 16 KB read per group of
//     1024 cycles of MMAs; the other way round, 256 rows by 128 outputs, more than L2 gives an SM).
//   warp 0       issues the copies: a ring of groups (rows, codes)
//   warps 1, 2   issue the MMAs, a half each: a group into one of three accumulators of 128 columns.  (Waits, issue and a commit take a warp some 600
//                cycles, more than the MMAs; one commit tells all who wait for a half, since each takes 50 to 150.)
//   warps 4-7    codes to bfloat16, one group of one half into one of two operand areas of tensor memory (64 columns each)
//   warps 8-15   take the accumulators out; each four warps have half of the rows
// Tiles are dealt out, cut along K and joined as those of the other types are (grouped_common.cuh).
// A group takes 1.04 us at 128 rows (2000 cycles; 1060 of MMAs) and hardly less at 32.  MMAs wait for accumulators to be taken out: the warps that do are busy 1700
// of the 2000 cycles, though their loads and additions by themselves take 330.  8192 rows of 5120 to 17920 take 1420 us one launch after the other (1.06 PFLOP/s;
// the operations' floor is 929), 1620 among passes that change their inputs; without the additions 1350, without unpacking 1335, with one MMA of eight 1400,
// without all three 1044, without the loads in front of the additions too 930.  What did not help: eight warps that unpack (those that take sums out then have
// 168 registers instead of 184: 1750 us); longer waits per poll (1520); additions that are not packed (1470); a half's sums by four warps of all rows
// instead of eight of half of them (1413, but three accumulators then need six barriers).
// A tile costs the same however few its rows and outputs are: of a plain product whose outputs leave up to 128 for the last column tile, that tile's
// second half is unpacked, multiplied and taken out for nothing.  (Compiled for 128 registers, the kernel spills 20 bytes a thread.)
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "gemv_common.cuh"
#include "grouped_common.cuh"
#include "int4_codes.cuh"

namespace {

constexpr int IM_STAGES = 4;
constexpr int IM_BOX = 32;                          // rows per copy
constexpr int IM_SUMS = 3;                          // accumulators
constexpr int IM_HALF = GP_COLS / 2;                // outputs of a half
constexpr int IM_X_BYTES = GP_ROWS * DIP_INT4_GROUP * 2, IM_CODE_BYTES = GP_COLS * DIP_INT4_GROUP / 2;
constexpr int IM_OPERAND = IM_SUMS * GP_ROWS, IM_OPERAND_COLS = DIP_INT4_GROUP / 2;     // columns of tensor memory: first of the operands; of one
static_assert(IM_OPERAND + 2 * IM_OPERAND_COLS == GP_TMEM_COLS, "fits tensor memory");
// Groups' worth of time that a cut tile's parts take to meet (8 us and more; with 4 or 30 instead no case changed by more than 3 %).
constexpr int IM_JOIN = 12;

template <bool GATED_> struct ManyKind {
    static constexpr bool GATED = GATED_, PAIR = false;
    static constexpr int TILE_ROWS = GP_ROWS;
    static constexpr int OUT_WARPS = 8, THREADS = (8 + OUT_WARPS) * 32;
    // registers of a thread: of the first four warps, of those that unpack codes, of the others (in all 504 of the launch's 512 per four)
    static constexpr int REGS_FEW = 48, REGS_CODES = 88, REGS_MANY = 184;
};

struct __align__(1024) ManySmem {
    unsigned char x[IM_STAGES][2][IM_X_BYTES / 2];      // 64 inputs each
    unsigned char codes[IM_STAGES][2][IM_CODE_BYTES / 2];
    __half scales[2 * IM_STAGES][2][IM_HALF];       // (twice the stages: the sums are taken out up to three halves behind the MMAs that free a stage)
    uint64_t full[IM_STAGES], scales_full[2 * IM_STAGES];    // a group's copies have landed
    uint64_t operand_full[2];
    uint64_t done[IM_STAGES][2];                    // a half's MMAs are through: its sums may be taken out, its operand and its copies replaced
    uint64_t sum_empty[IM_SUMS];
    uint64_t drained[2];
    uint32_t tmem_base;
    int last;
    int fail, peer_fail;
    int issued;                                     // groups that warp 0 has asked for
    GroupedPlan plan;
};

__device__ __forceinline__ void tmem_st(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
                 "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
                   "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
                   "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
                   "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
                 : "memory");
}

// Neighbouring bytes (whole pieces of 16) to shared memory.
__device__ __forceinline__ void bulk_load(void *dst, const void *src, unsigned bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

// D += A B with A in tensor memory.
__device__ __forceinline__ void many_mma(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t shape, uint32_t accumulate)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b), "r"(shape), "r"(accumulate) : "memory");
}

// A row's output: binary32, or rounded once to bfloat16.  (h is always: it is an operand of the next product, whose MMAs take no more.)
__device__ __forceinline__ void put(void *out, size_t at, float v, int out_f32)
{
    if (out_f32) static_cast<float *>(out)[at] = v;
    else static_cast<__nv_bfloat16 *>(out)[at] = __float2bfloat16_rn(v);
}

template <class K>
__device__ __forceinline__ void many_take(const GroupedParams &p, ManySmem &s, const Schedule<K> &plan, const Run &r, uint32_t lanes, int share,
                                          int place, int &buf, int &g)
{
    constexpr bool GATED = K::GATED;
    constexpr int N = GP_ROWS / 2, L = 16;           // rows of a thread, at most; columns that are loaded together
    const int lane = threadIdx.x & 31, per = (r.rows + 15) / 16 * 8, t0 = share * per, rows = min(per, r.rows - t0);      // (may be none)
    const int o = r.out0 + place;                    // gate/up: of both; plain: the second one's is IM_HALF further on
    float acc[2][N];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < N; ++j) acc[h][j] = 0.f;
    for (int k = r.k0; k < r.k1; ++k, ++g) {
        const int st = g % IM_STAGES, slot = g % (2 * IM_STAGES);
        const unsigned through = (g / IM_STAGES) & 1;
        wait_on(smem_u32(&s.scales_full[slot]), (g / (2 * IM_STAGES)) & 1, s, p.status, p.wait_limit_ns);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float scale = __half2float(s.scales[slot][h][place]) * INT4_PRODUCT;
            wait_on(smem_u32(&s.done[st][h]), through, s, p.status, p.wait_limit_ns);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t from = lanes + buf * GP_ROWS + t0;
            // one load is under way while the one in front is added
            uint32_t v[2][L];
            tmem_ld(from, v[0]);
#pragma unroll
            for (int c = 0; c < N / L; ++c)
                if (L * c < per) {
                    tmem_wait(v[c & 1]);
                    if (L * (c + 1) < per) tmem_ld(from + L * (c + 1), v[(c + 1) & 1]);
#pragma unroll
                    for (int j = 0; j < L; j += 2) fma2(acc[h][L * c + j], acc[h][L * c + j + 1], v[c & 1][j], v[c & 1][j + 1], scale);
                }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            arrive_first<false>(smem_u32(&s.sum_empty[buf]), lane);
            buf = buf == IM_SUMS - 1 ? 0 : buf + 1;
        }
    }

    if (r.k1 - r.k0 < p.steps) {
        // a part of the tile: the last of its blocks goes on with the sum of all.  Parts are [row][256 sums]
        const size_t mine = (size_t)t0 * GP_COLS + place;
        float *to = p.partials + plan.part_at(plan.block(), r.rest) + mine;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < rows) {
                to[j * GP_COLS] = acc[0][j];
                to[j * GP_COLS + IM_HALF] = acc[1][j];
            }
        int b0, b1;
        if (!part_is_last(p, s, plan, r, b0, b1)) return;
#pragma unroll
        for (int j = 0; j < N; ++j) acc[0][j] = acc[1][j] = 0.f;
        for (int b = b0; b <= b1; ++b) {
            const float *part = p.partials + plan.part_at(b, r.rest) + mine;
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < rows) {
                    acc[0][j] += __ldcg(part + j * GP_COLS);
                    acc[1][j] += __ldcg(part + j * GP_COLS + IM_HALF);
                }
        }
    }

    const size_t at = (size_t)(r.row0 + t0) * p.d_out + o;
    if (GATED) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < rows && o < p.d_out) put(p.out, at + (size_t)j * p.d_out, silu_f32(acc[0][j]) * acc[1][j], 0);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < rows) {
                if (o < p.d_out) put(p.out, at + (size_t)j * p.d_out, acc[0][j], p.out_f32);
                if (o + IM_HALF < p.d_out) put(p.out, at + IM_HALF + (size_t)j * p.d_out, acc[1][j], p.out_f32);
            }
    }
}

template <class K>
__global__ void __launch_bounds__(K::THREADS, 1)
int4_many_kernel(const __grid_constant__ CUtensorMap rows_map, const __grid_constant__ CUtensorMap w_map,
                 const __grid_constant__ CUtensorMap w2_map, const GroupedParams p)
{
    constexpr bool GATED = K::GATED;
    extern __shared__ unsigned char im_smem_raw[];
    ManySmem &s = *reinterpret_cast<ManySmem *>((reinterpret_cast<uintptr_t>(im_smem_raw) + 1023) & ~(uintptr_t)1023);
    DIP_TRACE_MIN(p.tr, 0);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem_base)), "n"(GP_TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 0) {
        for (int i = 0; i < IM_STAGES; ++i) {
            mbar_init(&s.full[i], 1);
            mbar_init(&s.scales_full[2 * i], 1);
            mbar_init(&s.scales_full[2 * i + 1], 1);
            mbar_init(&s.done[i][0], 1);
            mbar_init(&s.done[i][1], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s.operand_full[i], 4);
            mbar_init(&s.drained[i], 1);
        }
        for (int i = 0; i < IM_SUMS; ++i) mbar_init(&s.sum_empty[i], K::OUT_WARPS);
        s.fail = s.peer_fail = s.issued = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&rows_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&w_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&w2_map) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const Schedule<K> plan = {p, s.plan};
    dip_grid_dependency_wait();
    DIP_TRACE_MIN(p.tr, 1);
    if (warp == 0) {
        __syncwarp();
        grouped_plan(p, plan.ROWS, s.plan);
        __syncwarp();
        if (lane == 0) plan.divide();
        __syncwarp();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (warp == 0) asm volatile("barrier.cta.arrive 2, %0;" ::"n"(K::THREADS) : "memory");       // (goes on to its copies)
    else asm volatile("barrier.cta.sync 2, %0;" ::"n"(K::THREADS) : "memory");
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    dip_launch_dependents();
    const uint32_t tmem = s.tmem_base;               // (warp 0 has no use for it)
    bool failed = false;

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(K::REGS_FEW));
        if (warp == 0) {
            Run r;
            int g = 0;                               // groups so far
            for (int i = 0; !failed && plan.get(i, r); ++i) {
                const int boxes = (r.rows + IM_BOX - 1) / IM_BOX, w_row = r.expert * p.d_out + r.out0;
                // scales of the halves' outputs that there are
                const unsigned some0 = min(IM_HALF, p.d_out - r.out0) * 2, some1 = GATED ? some0 : max(0, min(IM_HALF, p.d_out - r.out0 - IM_HALF)) * 2;
                const unsigned bytes = IM_CODE_BYTES + boxes * IM_BOX * DIP_INT4_GROUP * 2;
                const __half *scales = static_cast<const __half *>(static_cast<const void *>(p.w_scales)), *scales1 = scales + IM_HALF;
                if (GATED) scales1 = static_cast<const __half *>(static_cast<const void *>(p.up_scales));
                size_t from = ((size_t)r.expert * p.steps + r.k0) * p.d_out + r.out0;
                for (int k = r.k0; k < r.k1; ++k, ++g, from += p.d_out) {
                    const int st = g % IM_STAGES;
                    if (g >= IM_STAGES && (!warp_wait(&s.done[st][0], (g / IM_STAGES - 1) & 1, p.wait_limit_ns) ||
                                           !warp_wait(&s.done[st][1], (g / IM_STAGES - 1) & 1, p.wait_limit_ns))) {
                        failed = true;
                        break;
                    }
                    if (elect_one()) {
                        mbar_expect_tx(&s.full[st], bytes);
                        const int slot = g % (2 * IM_STAGES);
                        mbar_expect_tx(&s.scales_full[slot], some0 + some1);
                        bulk_load(s.scales[slot][0], scales + from, some0, &s.scales_full[slot]);
                        if (some1) bulk_load(s.scales[slot][1], scales1 + from, some1, &s.scales_full[slot]);
                        tma_load<false>(s.codes[st][0], &w_map, k * (DIP_INT4_GROUP / 2), w_row, &s.full[st]);
                        tma_load<false>(s.codes[st][1], &w2_map, k * (DIP_INT4_GROUP / 2), GATED ? w_row : w_row + IM_HALF, &s.full[st]);
                        for (int b = 0; b < boxes; ++b) {
                            tma_load<false>(s.x[st][0] + b * IM_BOX * 128, &rows_map, k * DIP_INT4_GROUP, r.row0 + b * IM_BOX, &s.full[st]);
                            tma_load<false>(s.x[st][1] + b * IM_BOX * 128, &rows_map, k * DIP_INT4_GROUP + 64, r.row0 + b * IM_BOX, &s.full[st]);
                        }
                    }
                    __syncwarp();
                }
            }
            if (lane == 0) s.issued = g;
        } else if (warp <= 2) {
            const int h = warp - 1;
            const uint32_t a = tmem + IM_OPERAND + h * IM_OPERAND_COLS;
            const bool elected = elect_one();
            Run r;
            int g = 0, buf = h;                      // groups so far; the next accumulator: halves take them in turn
            unsigned phase = 1;                      // of its last release (the first three need none)
            for (int i = 0; !failed && plan.get(i, r); ++i) {
                const uint32_t shape = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)((r.rows + 15) / 16 * 2) << 17) | (8u << 24);
                for (int k = r.k0; k < r.k1; ++k, ++g) {
                    const int st = g % IM_STAGES;
                    if ((2 * g + h >= IM_SUMS && !warp_wait(&s.sum_empty[buf], phase, p.wait_limit_ns)) ||
                        !warp_wait(&s.full[st], (g / IM_STAGES) & 1, p.copy_wait_ns) || !warp_wait(&s.operand_full[h], g & 1, p.wait_limit_ns)) {
                        failed = true;
                        break;
                    }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t b0 = operand_desc(s.x[st][0]), b1 = operand_desc(s.x[st][1]);
                    const uint32_t to = tmem + buf * GP_ROWS;
                    if (elected) {
#pragma unroll
                        for (int q = 0; q < 8; ++q)              // 16 inputs each
                            many_mma(to, a + 8 * q, (q < 4 ? b0 : b1) + 2 * (q & 3), shape, q ? 1u : 0u);
                        grouped_commit<false>(&s.done[st][h]);
                    }
                    __syncwarp();
                    buf += 2;
                    if (buf >= IM_SUMS) {
                        buf -= IM_SUMS;
                        phase ^= 1u;
                    }
                }
            }
        }
        if (failed) {
            *(volatile int *)&s.fail = 1;
            atomicExch(p.status, 1);
        }
        // All roles are through.  Where any wait has run out, MMAs and copies may still be under way: they are waited for.
        roles_end<false, K::THREADS>(s, tid);
        if (gave_up<false>(s)) {
            if (warp == 1 || warp == 2) {
                if (elect_one()) grouped_commit<false>(&s.drained[warp - 1]);
                __syncwarp();
                warp_wait(&s.drained[warp - 1], 0, p.wait_limit_ns);
            }
            if (warp == 0) {
                drain_copies<IM_STAGES, false>(s.full, s.issued, 0, [](int) { return 0u; }, p.wait_limit_ns);
                drain_copies<2 * IM_STAGES, false>(s.scales_full, s.issued, 0, [](int) { return 0u; }, p.wait_limit_ns);
            }
        }
    } else if (warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(K::REGS_CODES));
        const int place = (warp & 3) * 32 + lane;    // lane of tensor memory
        const uint32_t to = tmem + ((uint32_t)((warp & 3) * 32) << 16) + IM_OPERAND;
        // a half's stores are through: the MMAs may have it
        const auto hand_over = [&](int h) {
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            arrive_first<false>(smem_u32(&s.operand_full[h]), lane);
        };
        Run r;
        int g = 0;
        for (int i = 0; plan.get(i, r); ++i) {
            for (int k = r.k0; k < r.k1; ++k, ++g) {
                const int st = g % IM_STAGES;
                wait_on(smem_u32(&s.full[st]), (g / IM_STAGES) & 1, s, p.status, p.wait_limit_ns);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const unsigned char *row = s.codes[st][h] + place * (DIP_INT4_GROUP / 2);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t v[32];
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            // (64-byte swizzle)
                            const uint4 w = *reinterpret_cast<const uint4 *>(row + (((2 * c + q) ^ (place >> 1 & 3)) << 4));
                            int4_in_order(w.x, v + 16 * q);
                            int4_in_order(w.y, v + 16 * q + 4);
                            int4_in_order(w.z, v + 16 * q + 8);
                            int4_in_order(w.w, v + 16 * q + 12);
                        }
                        if (c == 0) {
                            // (the half in front, whose stores have had the time of this one's first)
                            if (h == 1) hand_over(0);
                            if (g >= 1) wait_on(smem_u32(&s.done[(g - 1) % IM_STAGES][h]), ((g - 1) / IM_STAGES) & 1, s, p.status, p.wait_limit_ns);
                            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        }
                        tmem_st(to + h * IM_OPERAND_COLS + 32 * c, v);
                    }
                }
                hand_over(1);
            }
        }
        roles_end<false, K::THREADS>(s, tid);
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(K::REGS_MANY));
        const int share = (warp - 8) >> 2, place = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        int buf = 0, g = 0;                          // accumulator, groups so far
        Run r;
        for (int i = 0; plan.get(i, r); ++i) many_take<K>(p, s, plan, r, lanes, share, place, buf, g);
        roles_end<false, K::THREADS>(s, tid);
    }
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(GP_TMEM_COLS) : "memory");
    DIP_TRACE_MAX(p.tr, 2);
}

// Pieces of `box` rows by `width` items of a row-major [n][d] matrix of items of one or two bytes; zeros outside.
bool encode(CUtensorMap *map, const void *p, int item, size_t n, int d, int width, int box, CUtensorMapSwizzle swizzle)
{
    const cuuint64_t dims[2] = {(cuuint64_t)d, (cuuint64_t)n}, strides[1] = {(cuuint64_t)d * item};
    const cuuint32_t piece[2] = {(cuuint32_t)width, (cuuint32_t)box}, one[2] = {1, 1};
    return encoder()(map, item == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(p), dims,
                     strides, piece, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class K>
cudaError_t launch(dip_ctx *ctx, int ctas, cudaStream_t stream, const CUtensorMap (&m)[3], const GroupedParams &p)
{
    static dip_per_device_once once;
    const auto kernel = int4_many_kernel<K>;
    const size_t smem = sizeof(ManySmem) + 1024;
    static_assert(sizeof(ManySmem) + 1024 <= 227 * 1024, "fits a CTA's shared memory");
    // (the warps that take sums out would wait for ever for registers that the launch does not have)
    static const bool enough = [&] {
        cudaFuncAttributes a;
        return cudaFuncGetAttributes(&a, kernel) == cudaSuccess &&
               a.numRegs * (8 + K::OUT_WARPS) >= K::REGS_FEW * 4 + K::REGS_CODES * 4 + K::REGS_MANY * K::OUT_WARPS;
    }();
    if (!enough) return cudaErrorLaunchOutOfResources;
    const cudaError_t e = dip_raise_smem_limit(once, ctx->device, kernel, smem);
    if (e != cudaSuccess) return e;
    return dip_launch_pdl(kernel, dim3(ctas), dim3(K::THREADS), smem, stream, m[0], m[1], m[2], p);
}

}  // namespace

dip_status dip_launch_int4_many(dip_ctx *ctx, const dip_grouped_matrix &w, const dip_grouped_matrix *up, const void *rows, int n_rows,
                                const int32_t *offset, void *out, bool out_f32, cudaStream_t stream)
{
    const size_t w_rows = (size_t)w.n_experts * w.d_out;
    CUtensorMap maps[3];
    if (!encoder() || !encode(&maps[0], rows, 2, n_rows, w.d_in, 64, IM_BOX, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !encode(&maps[1], w.values, 1, w_rows, w.d_in / 2, DIP_INT4_GROUP / 2, IM_HALF, CU_TENSOR_MAP_SWIZZLE_64B) ||
        !encode(&maps[2], up ? up->values : w.values, 1, w_rows, w.d_in / 2, DIP_INT4_GROUP / 2, IM_HALF, CU_TENSOR_MAP_SWIZZLE_64B)) {
        snprintf(ctx->err, sizeof(ctx->err), "cuTensorMapEncodeTiled failed");
        return DIP_ERR_CUDA;
    }
    const int width = up ? GP_COLS / 2 : GP_COLS, met = min(w.n_experts, n_rows);
    GroupedParams p = {};
    p.w_scales = static_cast<const float *>(w.scales);            // (binary16: what reads them knows)
    p.up_scales = up ? static_cast<const float *>(up->scales) : nullptr;
    p.n_experts = w.n_experts;
    p.d_out = w.d_out;
    p.d_in = w.d_in;
    p.n_rows = n_rows;
    p.steps = (w.d_in + DIP_INT4_GROUP - 1) / DIP_INT4_GROUP;
    p.n_cols = (w.d_out + width - 1) / width;
    p.join = IM_JOIN;
    p.offset = offset;
    p.out = out;
    p.out_f32 = out_f32;
    p.partials = ctx->partials;
    p.tickets = ctx->group_tickets;
    p.status = ctx->status;
    p.copy_wait_ns = ctx->wait_limit_ns;
    p.wait_limit_ns = ctx->block_wait_ns;
    p.tr = dip_trace_slot(ctx, up ? 10 : 11);
    const long long tiles = (long long)((n_rows + GP_ROWS - 1) / GP_ROWS + met - 1) * p.n_cols;
    const int ctas = (int)min((long long)ctx->sm_count, max(tiles, tiles * p.steps / GP_MIN_STEPS));
    DIP_CUDA_TRY(ctx, up ? launch<ManyKind<true>>(ctx, ctas, stream, maps, p) : launch<ManyKind<false>>(ctx, ctas, stream, maps, p));
    return DIP_OK;
}
