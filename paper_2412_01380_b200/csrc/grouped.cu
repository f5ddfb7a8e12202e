// Products of groups of rows, a group per expert, on the fifth-generation tensor cores: y[r] = W[e(r)] rows[r], and
// h[r] = silu(Wg[e(r)] rows[r]) * (Wu[e(r)] rows[r]).  One kernel for a token's one or two rows and for a prompt's thousands.
//
// A block's tile is 128 rows of one expert by 256 rows of its weights (gate/up: the 128 gate and the 128 up rows of the same
// outputs, so that one thread has both).  Both operands are K-major 128-byte pieces (64 bfloat16, 128 e4m3) that TMA lays
// into shared memory with the 128-byte swizzle the operand descriptors name.
//   PAIR   two blocks of a cluster share a tile of 256 rows: each loads its 128 rows and half of the weights, and the first one's
//          MMAs (cta_group::2, M = 256) read both halves.  Per step and SM 32 KB come in and 32 KB are read, which shared
//          memory does in the 512 cycles that the MMAs take.  (Alone it is 48 and 48 KB: 768 cycles, measured 785.)
//   whole  a block by itself.
//   few    the same for groups of few rows, tiles of at most 64: the operands change their roles.  The weights are the M side (two
//          MMAs of 128) and the rows the N side, as many columns as there are rows (in sixteens).  The loads are alike, but a thread then
//          has one output of a few rows instead of one row of 64 outputs, and what follows the last step takes as long as there are rows.
//   warp 0      issues the copies: a ring of steps
//   warp 1      issues the MMAs (N = 256, four per step) into one of two accumulators of 256 columns; SPLIT: warps 1 and 2 those of
//               a half each
//   warp 3      FP8: brings the rows' scales, eight steps at a time, into a ring of their own
//   the others  take the accumulators out: thread = row, and each four warps have a share of the columns
// BF16: an accumulator is a tile, and the next tile's MMAs run while the first is taken out.  FP8: a step is a block of 128
// input indices, which has scales of its own, so every step's accumulator is taken out and added, times row scale * weight
// scale, to binary32 sums in registers: 256 columns per warp scheduler and step against the 512 cycles of its MMAs.
//
// Blocks stay: whole rounds of tiles are dealt out one to a block (or pair), and what is left over (all of it where there are
// fewer tiles than SMs, as for a token) is cut along K into equal runs of steps, one per block, in tile order.  A tile's
// parts meet in the partial sums' workspace; the block that comes last adds them up in order of K, so results do not
// depend on who that is, and nobody waits.
#include <cuda.h>
#include <cuda_bf16.h>

#include "common.cuh"
#include "float8.cuh"
#include "gemv_common.cuh"

namespace {

constexpr int GP_ROWS = DIP_GROUP_ROWS, GP_COLS = DIP_GROUP_COLS;
constexpr int GP_STEP_BYTES = 128;                  // of a row, per step
constexpr int GP_BOX = 32;                          // rows per copy of the rows of a tile of few
constexpr int GP_A_BYTES = GP_ROWS * GP_STEP_BYTES, GP_B_BYTES = GP_COLS * GP_STEP_BYTES;
constexpr int GP_TMEM_COLS = 512;
constexpr int GP_MIN_STEPS = 4;                     // a part of a tile has at least so many
// Steps' worth of time that a cut tile's parts take to meet: written, counted, read and added (7 us for a tile of 128 rows; 3.5 us for one row,
// and as many steps more as there are rows.  8 rows each for 16 experts, 4096 to 2048, bfloat16: 50.7 us with whole tiles, 56.5 cut).
// One constant for both types, though their steps do not take the same time.
constexpr int GP_JOIN_FEW = 8, GP_JOIN = 20;
constexpr int GP_TWO_RUNS = 6;                      // steps' worth of time that a block loses between two runs
constexpr int GP_SCALE_STEPS = 8, GP_SCALE_SLOTS = 4;   // steps of scales that come together, and how many such groups there is room for
constexpr int GP_FEW = 64;                          // rows of a tile that are columns of its sums
constexpr int GP_CHUNK = 12;                        // row tiles that go through an expert's weights together
enum { GP_FEW_ROWS, GP_WHOLE, GP_PAIR };            // see above
template <bool FP8_, bool GATED_, int MODE> struct Kind {
    static constexpr bool FP8 = FP8_, GATED = GATED_, PAIR = MODE == GP_PAIR, FEW = MODE == GP_FEW_ROWS;
    static constexpr int TILE_ROWS = PAIR ? 2 * GP_ROWS : FEW ? GP_FEW : GP_ROWS;
    static constexpr int A_BYTES = (FEW ? GP_FEW : GP_ROWS) * GP_STEP_BYTES, B_BYTES = PAIR ? GP_B_BYTES / 2 : GP_B_BYTES;
    // (few rows, bytes of weights in flight: 128 KB and 160 are 27 and 31 us for one 8-bit row of 5120 to 17920, 49.5 and 48.7 us for
    // two bfloat16 rows of 4096 to 14336)
    static constexpr int STAGES = PAIR || (FEW && !FP8) ? 5 : 4;
    static constexpr int PIECE = PAIR ? 64 : 32;     // bytes of a row that leave together
    // 8-bit pairs make and take out a step's accumulator in halves, with a warp for each half's MMAs: one warp that waits for two halves
    // and issues both needs some 900 cycles a step, and the way from an MMA by its warps' registers back to the next MMA into the
    // same columns, across the pair, has two steps to fit into.  The halves read the rows twice: 80 KB of shared memory per step, 640
    // cycles.
    static constexpr bool SPLIT = FP8 && PAIR;
    // Warps that take sums out.  FP8 keeps a tile's sums in registers over all steps, and two warps per scheduler with 128 of them
    // each can have two loads of 32 accumulator columns in hand; BF16 only has to get rid of a tile.
    static constexpr int OUT_WARPS = FP8 || FEW ? 8 : 16, THREADS = (4 + OUT_WARPS) * 32;
    // registers of a thread of the first four warps and of the others; in all what the launch has:
    // (56 + 2 * 224) / 3 = (40 + 2 * 232) / 3 = 168 each, or (64 + 4 * 104) / 5 = 96
    static constexpr int REGS_FEW = FP8 ? (PAIR ? 56 : 40) : 64, REGS_MANY = FP8 ? (PAIR ? 224 : 232) : 104;
};

struct GroupedParams {
    const float *w_scales, *up_scales, *row_scales;
    int n_experts, d_out, d_in, n_rows, steps, n_cols, join;
    const int32_t *offset;
    void *out;
    float *out_scales;
    int out_f32;
    float *partials;
    unsigned int *tickets;
    int *status;
    unsigned long long copy_wait_ns, wait_limit_ns;      // on a copy; on other warps
    unsigned long long *tr;
};

struct GroupedPlan {
    int start[DIP_MAX_EXPERTS + 1];                 // first row of each expert
    int tiles[DIP_MAX_EXPERTS + 1];                 // row tiles in front of it
    int whole;                                      // rounds of whole tiles
    int units, parts;                               // steps of the tiles that are cut, blocks that share them
};

template <class K>
struct __align__(1024) GroupedSmem {
    static constexpr bool RING = K::FP8 && !K::FEW;
    unsigned char a[K::STAGES][K::A_BYTES];
    unsigned char b[K::STAGES][K::B_BYTES];
    unsigned char out[K::FEW ? 1 : K::OUT_WARPS][32 * K::PIECE];
    uint64_t full[K::STAGES], empty[K::STAGES];     // a step's copies have landed; its MMAs have read them
    uint64_t sum_full[2][2], sum_empty[2][2];       // an accumulator (SPLIT: a half of it) is complete; has been taken out
    uint64_t scale_full[GP_SCALE_SLOTS], scale_empty[GP_SCALE_SLOTS];
    uint64_t drained[2];
    float row_scale[RING ? GP_SCALE_SLOTS * GP_SCALE_STEPS : 1][RING ? GP_ROWS : 1];
    float2 w_scale[GP_SCALE_SLOTS * GP_SCALE_STEPS];     // of a tile's two blocks of weights (gate/up: one of each)
    uint32_t tmem_base;
    int last;
    int fail, peer_fail;                            // a wait of this block (PAIR: of the other one) has run out
    int issued;                                     // steps that warp 0 has asked for
    float amax[4 * GP_ROWS];
    GroupedPlan plan;
};

// PAIR: into this block's shared memory, counted by the first block's barrier (whose address has the block's bit clear).
template <bool PAIR>
__device__ __forceinline__ void tma_load(void *dst, const CUtensorMap *map, int x, int y, uint64_t *bar)
{
    if (PAIR)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar) & 0xfeffffffu) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void tma_prefetch(const CUtensorMap *map, int x, int y)
{
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}

// Four bytes to shared memory, asynchronously.
__device__ __forceinline__ void copy4(float *dst, const float *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

// Whether the phase with the given parity is through (waits a little if it is not).
__device__ __forceinline__ bool try_wait(uint32_t bar, unsigned parity)
{
    unsigned ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0u;
}

// A whole warp's bounded wait: all lanes go on alike.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, unsigned parity, unsigned long long limit_ns)
{
    if (__all_sync(0xffffffffu, try_wait(smem_u32(bar), parity))) return true;
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, limit_ns));
}

// The same for those who go on in any case: once a wait has run out, s.fail says so to the others, and nothing waits any more.
// (What a step costs these warps beside its arithmetic is what bounds 8-bit products; they have no control flow for failures.)
template <typename Smem>
__device__ __forceinline__ void wait_on(uint32_t bar, unsigned parity, Smem &s, int *status, unsigned long long limit_ns)
{
    if (!try_wait(bar, parity)) {
        unsigned long long t0 = 0;
        for (unsigned i = 1; !*(volatile int *)&s.fail && !try_wait(bar, parity); ++i) {
            if (i & 63u) continue;
            const unsigned long long now = dip_gtime();
            if (t0 == 0) {
                t0 = now;
            } else if (now - t0 > limit_ns) {
                *(volatile int *)&s.fail = 1;
                atomicExch(status, 1);
                break;
            }
        }
    }
    __syncwarp();
}

// One lane of a whole warp.  (A role's warp goes through its loop as a whole and elects a lane where it issues: with the loop in
// a branch of lane 0, whose operands the compiler cannot know to be uniform, a copy took 180 cycles to issue and an MMA 100.)
__device__ __forceinline__ bool elect_one()
{
    unsigned yes;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(yes));
    return yes != 0u;
}

// K-major operand, 128-byte swizzle: groups of 8 rows are 1 KB apart.
__device__ __forceinline__ uint64_t operand_desc(const void *p)
{
    return (uint64_t)((smem_u32(p) & 0x3ffffu) >> 4) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// Instruction descriptor: binary32 sums, K-major operands of M = 128 (PAIR: 256) and N = n; bfloat16 or e4m3
template <bool FP8, bool PAIR>
__device__ __forceinline__ uint32_t grouped_shape(int n)
{
    return (1u << 4) | (FP8 ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)(n >> 3) << 17) | ((PAIR ? 16u : 8u) << 24);
}

template <bool FP8, bool PAIR>
__device__ __forceinline__ void grouped_mma(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t shape, uint32_t accumulate)
{
#define GP_MMA(group, kind)                                                                                                         \
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::" group ".kind::" kind " [%0], %1, %2, %3, p;\n}" \
                 ::"r"(d_tmem), "l"(a), "l"(b), "r"(shape), "r"(accumulate) : "memory")
    if (FP8 && PAIR) GP_MMA("2", "f8f6f4");
    else if (FP8) GP_MMA("1", "f8f6f4");
    else if (PAIR) GP_MMA("2", "f16");
    else GP_MMA("1", "f16");
#undef GP_MMA
}

// Arrives at the barrier (PAIR: at both blocks') once the MMAs so far are through.
template <bool PAIR>
__device__ __forceinline__ void grouped_commit(uint64_t *bar)
{
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// One lane of the warp arrives at the first block's barrier.  (Predicated: a branch and its way back together took 190 cycles.)
template <bool PAIR>
__device__ __forceinline__ void arrive_first(uint32_t bar, int lane)
{
    if (PAIR)
        asm volatile("{\n .reg .pred p;\n .reg .b32 r;\n setp.eq.s32 p, %1, 0;\n mapa.shared::cluster.u32 r, %0, 0;\n"
                     " @p mbarrier.arrive.shared::cluster.b64 _, [r];\n}" ::"r"(bar), "r"(lane) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.eq.s32 p, %1, 0;\n @p mbarrier.arrive.shared::cta.b64 _, [%0];\n}"
                     ::"r"(bar), "r"(lane) : "memory");
}

__device__ __forceinline__ void pair_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A word of the other block's shared memory.
__device__ __forceinline__ uint32_t peer_word(const void *p)
{
    uint32_t a;
    asm("{\n .reg .b32 r;\n mov.u32 r, %%cluster_ctarank;\n xor.b32 r, r, 1;\n mapa.shared::cluster.u32 %0, %1, r;\n}" : "=r"(a) : "r"(smem_u32(p)));
    return a;
}
__device__ __forceinline__ int peer_load(const int *p)
{
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(peer_word(p)) : "memory");
    return v;
}
__device__ __forceinline__ void peer_store(int *p, int v) { asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(peer_word(p)), "r"(v) : "memory"); }

// As many bytes less for the phase to wait for.
__device__ __forceinline__ void mbar_complete_tx(uint64_t *bar, unsigned bytes)
{
    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}

// A wait has run out, and no copy may be on its way into a block that leaves: one warp (PAIR: of the first block) waits for the
// steps whose copies may not have landed.  A stage is asked for again only when its step has been read, so they are the last
// STAGES.  No more copies are issued (a block barrier is behind; PAIR: one of both blocks).
// mine, other: steps that this block and the second one have asked for.  Where one was ahead of the other, a step's barrier expects
// copies that nobody asks for any more, or does not know yet of the second block's: second_bytes(j) says how many bytes those of step j are.
template <int STAGES, bool PAIR, class Bytes>
__device__ __forceinline__ void drain_copies(uint64_t *full, int mine, int other, const Bytes &second_bytes, unsigned long long limit_ns)
{
    const int steps = PAIR ? max(mine, other) : mine;
    if (PAIR) {
        for (int j = min(mine, other); j < steps; ++j) {
            const unsigned bytes = second_bytes(j);
            if (elect_one()) {
                if (mine > other) mbar_complete_tx(&full[j % STAGES], bytes);
                else mbar_expect_tx(&full[j % STAGES], bytes);
            }
            __syncwarp();
        }
    }
    for (int j = max(0, steps - STAGES); j < steps; ++j) warp_wait(&full[j % STAGES], (j / STAGES) & 1, limit_ns);
}

// 8, 16 or 32 columns of this warp's 32 lanes: thread = lane, register = column.  The wait names the registers, so that nothing
// uses them before it.
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[8])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]),
                   "+r"(r[7])::"memory");
}
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]),
                   "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]),
                   "+r"(r[15])::"memory");
}
__device__ __forceinline__ void tmem_ld(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
                 "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
                   "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
                   "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]),
                   "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])::"memory");
}

// (a0, a1) += (d0, d1) * s, in one instruction.
__device__ __forceinline__ void fma2(float &a0, float &a1, uint32_t d0, uint32_t d1, float s)
{
    asm("{\n .reg .b64 a, d, f;\n mov.b64 a, {%0, %1};\n mov.b64 d, {%2, %3};\n mov.b64 f, {%4, %4};\n fma.rn.f32x2 a, d, f, a;\n"
        " mov.b64 {%0, %1}, a;\n}" : "+f"(a0), "+f"(a1) : "r"(d0), "r"(d1), "f"(s));
}

// Barrier of the warps that take sums out.
template <class K>
__device__ __forceinline__ void out_barrier() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(K::OUT_WARPS * 32) : "memory"); }

// One run of steps of one tile.
struct Run {
    int expert, row0, rows, out0;   // the tile: its first row, its rows, its first output
    int k0, k1;                     // steps
    int rest;                       // index among the tiles that are cut, -1: dealt out whole
};

// The runs of this block, in order.  Every role walks through them for itself, and keeps nothing of this in registers meanwhile.
// (32 bits hold it all: at most 2^21 tiles, and fewer than a block's worth of cut ones of at most 512 steps.)
template <class K>
struct Schedule {
    static constexpr bool GATED = K::GATED, PAIR = K::PAIR;
    static constexpr int ROWS = K::TILE_ROWS;
    const GroupedParams &p;
    volatile GroupedPlan &s;

    __device__ __forceinline__ int block() const { return PAIR ? blockIdx.x >> 1 : blockIdx.x; }
    __device__ __forceinline__ int blocks() const { return PAIR ? gridDim.x >> 1 : gridDim.x; }
    // by one thread, once the experts' rows and tiles are known
    __device__ __forceinline__ void divide() const
    {
        const int tiles = s.tiles[p.n_experts] * p.n_cols, whole = tiles / blocks(), rest = tiles - whole * blocks(), units = rest * p.steps;
        int parts = min(blocks(), max(units / GP_MIN_STEPS, rest));
        // runs within one tile each, where that makes them hardly longer: a block with two has a tile's end in the middle of its steps
        const int each = rest ? parts / rest : 1;
        if (parts > rest && (p.steps + each - 1) / each <= units / parts + GP_TWO_RUNS) parts = rest * each;
        if (parts > rest && units / parts + p.join >= p.steps) parts = rest;      // (they stay whole)
        s.whole = whole;
        s.units = units;
        s.parts = parts;
    }
    // the block that has a unit, and which of its runs is the one in cut tile `rest`
    __device__ __forceinline__ int block_of(int unit) const { return ((unit + 1) * s.parts - 1) / s.units; }
    __device__ __forceinline__ int run_of(int b, int rest) const { return s.units * b / s.parts / p.steps == rest ? 0 : 1; }
    // where block b (of this one's kind in its pair) leaves its part of the cut tile, in floats
    __device__ __forceinline__ size_t part_at(int b, int rest) const
    {
        return (size_t)(2 * (PAIR ? 2 * b + (int)(blockIdx.x & 1) : b) + run_of(b, rest)) * (GP_ROWS * GP_COLS);
    }

    __device__ __forceinline__ void locate(int tile, Run &r) const
    {
        int lo = 0, hi = p.n_experts;             // the expert with tiles[e] * p.n_cols <= tile < tiles[e + 1] * p.n_cols
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s.tiles[mid] * p.n_cols <= tile) lo = mid;
            else hi = mid;
        }
        const int n_rows = s.start[lo + 1] - s.start[lo], row_tiles = s.tiles[lo + 1] - s.tiles[lo];
        int in = tile - s.tiles[lo] * p.n_cols, m = 0, here = row_tiles;
        if (row_tiles > GP_CHUNK) {
            m = in / (GP_CHUNK * p.n_cols) * GP_CHUNK;
            in -= m * p.n_cols;
            here = min(GP_CHUNK, row_tiles - m);
        }
        const int col = here == 1 ? in : in / here;
        m += in - col * here;
        r.expert = lo;
        r.row0 = s.start[lo] + m * ROWS;
        r.rows = min(ROWS, n_rows - m * ROWS);
        r.out0 = col * (GATED ? GP_COLS / 2 : GP_COLS);
    }
    __device__ __forceinline__ bool get(int i, Run &r) const
    {
        const int whole = s.whole;
        r.rest = -1;
        r.k0 = 0;
        r.k1 = p.steps;
        int tile = i * blocks() + block();
        if (i >= whole) {
            const int units = s.units, parts = s.parts;
            if (block() >= parts) return false;
            int u = units * block() / parts;
            const int end = units * (block() + 1) / parts;
            for (i -= whole; i > 0 && u < end; --i) u = min(end, (u / p.steps + 1) * p.steps);
            if (u >= end) return false;
            r.rest = u / p.steps;
            r.k0 = u - r.rest * p.steps;
            r.k1 = min(p.steps, r.k0 + (end - u));
            tile = whole * blocks() + r.rest;
        }
        locate(tile, r);
        return true;
    }
};

// first rows and tiles of the experts, by one warp
__device__ __forceinline__ void grouped_plan(const GroupedParams &p, int tile_rows, GroupedPlan &s)
{
    const int lane = threadIdx.x & 31, each = (p.n_experts + 32) / 32;      // offsets per lane
    const int i0 = min(lane * each, p.n_experts + 1), i1 = min(i0 + each, p.n_experts + 1);
    int most = 0;
    for (int i = i0; i < i1; ++i) {
        const int v = p.offset ? min(p.offset[i], p.n_rows) : i ? p.n_rows : 0;
        most = max(most, v);
        s.start[i] = most;
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, most, o);
        if (lane >= o) most = max(most, v);
    }
    int before = __shfl_up_sync(0xffffffffu, most, 1);
    if (lane == 0) before = 0;
    for (int i = i0; i < i1; ++i) s.start[i] = max(s.start[i], before);
    __syncwarp();
    int n = 0;
    for (int i = i0; i < i1; ++i) {
        s.tiles[i] = n;
        if (i < p.n_experts) n += (s.start[i + 1] - s.start[i] + tile_rows - 1) / tile_rows;
    }
    int incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    for (int i = i0; i < i1; ++i) s.tiles[i] += incl - n;
}

// A part of a cut tile is in the workspace (this thread's share of it): true for the warps of the block that came last.
template <class K>
__device__ __forceinline__ bool part_is_last(const GroupedParams &p, GroupedSmem<K> &s, const Schedule<K> &plan, const Run &r, int &b0, int &b1)
{
    b0 = plan.block_of(r.rest * p.steps);
    b1 = plan.block_of((r.rest + 1) * p.steps - 1);
    __threadfence();
    out_barrier<K>();
    if (threadIdx.x == K::THREADS - 1) {
        unsigned int *ticket = p.tickets + (K::PAIR ? 2 * r.rest + (int)(blockIdx.x & 1) : r.rest);
        s.last = atomicAdd(ticket, 1u) == (unsigned)(b1 - b0);
        if (s.last) *ticket = 0u;
        __threadfence();
    }
    out_barrier<K>();
    return s.last != 0;
}

// The sums of a tile of few rows and what becomes of them: thread = output, values = rows.  Each four warps have a share of the rows; plain: the first or the second 128 outputs of a share; gate/up: a thread has gate and up of
// its output.
template <class K>
__device__ __forceinline__ void take_few(const GroupedParams &p, GroupedSmem<K> &s, const Schedule<K> &plan, const Run &r, uint32_t lanes,
                                         int share, int place, int &n)
{
    constexpr bool FP8 = K::FP8, GATED = K::GATED;
    constexpr int SHARES = K::OUT_WARPS / (GATED ? 4 : 8), N = GP_FEW / SHARES;         // rows of a thread: at most N
    const int lane = threadIdx.x & 31, per = ((r.rows + SHARES - 1) / SHARES + 7) / 8 * 8;
    const int t0 = (GATED ? share : share >> 1) * per, rows = min(per, r.rows - t0);      // (may be none)
    const int side = GATED ? 0 : GP_COLS / 2 * (share & 1), o = r.out0 + side + place;
    const uint32_t sums = lanes + side + t0;
    const int in_blocks = (p.d_in + DIP_FP8_BLOCK - 1) / DIP_FP8_BLOCK, out_blocks = (p.d_out + DIP_FP8_BLOCK - 1) / DIP_FP8_BLOCK;
    float a[N], u[GATED ? N : 1];
    if (FP8) {
#pragma unroll
        for (int j = 0; j < N; ++j) a[j] = 0.f;
        if (GATED) {
#pragma unroll
            for (int j = 0; j < N; ++j) u[j] = 0.f;
        }
        // a lane keeps the scales of row t0 + lane and of the one 32 behind it, and asks for the next step's in good time (plain loads: when
        // this kernel starts, the one in front may still be writing them)
        const float *xs = p.row_scales + (size_t)min(r.row0 + t0 + lane, r.row0 + r.rows - 1) * in_blocks;
        const float *ys = p.row_scales + (size_t)min(r.row0 + t0 + 32 + lane, r.row0 + r.rows - 1) * in_blocks;
        const size_t at = ((size_t)r.expert * out_blocks + min((r.out0 + side) / DIP_FP8_BLOCK, out_blocks - 1)) * in_blocks;
        const float *ws = p.w_scales + at, *us = GATED ? p.up_scales + at : ws;
        float next_x = xs[r.k0], next_w = __ldg(ws + r.k0), next_u = __ldg(us + r.k0), next_y = ys[r.k0];
        for (int k = r.k0; k < r.k1; ++k, ++n) {
            const float sx = next_x, sy = next_y, w = next_w, v = next_u;
            if (k + 1 < r.k1) {
                next_x = xs[k + 1];
                if (N > 32) next_y = ys[k + 1];
                next_w = __ldg(ws + k + 1);
                if (GATED) next_u = __ldg(us + k + 1);
            }
            const int buf = n & 1;
            wait_on(smem_u32(&s.sum_full[buf][0]), (n / 2) & 1, s, p.status, p.wait_limit_ns);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
            for (int c = 0; c < N / 8; ++c)
                if (8 * c < rows) {
                    uint32_t d[8], e[8];
                    tmem_ld(sums + buf * GP_COLS + 8 * c, d);
                    if (GATED) {
                        tmem_ld(sums + buf * GP_COLS + GP_COLS / 2 + 8 * c, e);
                        tmem_wait(e);
                    }
                    tmem_wait(d);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float x = __shfl_sync(0xffffffffu, c < 4 ? sx : sy, (8 * c + j) & 31);
                        a[8 * c + j] = fmaf(__uint_as_float(d[j]), x * w, a[8 * c + j]);
                        if (GATED) u[8 * c + j] = fmaf(__uint_as_float(e[j]), x * v, u[8 * c + j]);
                    }
                }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.sum_empty[buf][0]);
        }
    } else {
        const int buf = n & 1;
        wait_on(smem_u32(&s.sum_full[buf][0]), (n / 2) & 1, s, p.status, p.wait_limit_ns);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int c = 0; c < N / 8; ++c)
            if (8 * c < rows) {
                uint32_t d[8], e[8];
                tmem_ld(sums + buf * GP_COLS + 8 * c, d);
                if (GATED) {
                    tmem_ld(sums + buf * GP_COLS + GP_COLS / 2 + 8 * c, e);
                    tmem_wait(e);
                }
                tmem_wait(d);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    a[8 * c + j] = __uint_as_float(d[j]);
                    if (GATED) u[8 * c + j] = __uint_as_float(e[j]);
                }
            }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.sum_empty[buf][0]);
        ++n;
    }

    if (r.k1 - r.k0 < p.steps) {
        // a part of the tile: the last of its blocks goes on with the sum of all.  Parts are [row][256 sums]
        const size_t mine = (size_t)t0 * GP_COLS + side + place;
        float *to = p.partials + plan.part_at(plan.block(), r.rest) + mine;
#pragma unroll
        for (int c = 0; c < N / 8; ++c)
            if (8 * c < rows) {
#pragma unroll
                for (int j = 8 * c; j < 8 * c + 8; ++j)
                    if (j < rows) {
                        to[j * GP_COLS] = a[j];
                        if (GATED) to[j * GP_COLS + GP_COLS / 2] = u[j];
                    }
            }
        int b0, b1;
        if (!part_is_last(p, s, plan, r, b0, b1)) return;
#pragma unroll
        for (int j = 0; j < N; ++j) a[j] = 0.f;
        if (GATED) {
#pragma unroll
            for (int j = 0; j < N; ++j) u[j] = 0.f;
        }
        for (int b = b0; b <= b1; ++b) {
            const float *from = p.partials + plan.part_at(b, r.rest) + mine;
#pragma unroll
            for (int c = 0; c < N / 8; ++c)
                if (8 * c < rows) {
#pragma unroll
                    for (int j = 8 * c; j < 8 * c + 8; ++j)
                        if (j < rows) {
                            a[j] += __ldcg(from + j * GP_COLS);
                            if (GATED) u[j] += __ldcg(from + j * GP_COLS + GP_COLS / 2);
                        }
                }
        }
    }

    const bool there = o < p.d_out;
    const size_t at = (size_t)(r.row0 + t0) * p.d_out + o;
    if (GATED) {
#pragma unroll
        for (int c = 0; c < N / 8; ++c)
            if (8 * c < rows) {
#pragma unroll
                for (int j = 8 * c; j < 8 * c + 8; ++j) {
                    a[j] = silu_f32(a[j]) * u[j];
                    if (FP8) {
                        const unsigned most = __reduce_max_sync(0xffffffffu, there ? __float_as_uint(fmaxf(fabsf(a[j]), 0.f)) : 0u);
                        if (lane == 0) s.amax[(threadIdx.x >> 5 & 3) * GP_FEW + t0 + j] = __uint_as_float(most);
                    }
                }
            }
    }
    if (GATED && FP8) out_barrier<K>();
#pragma unroll
    for (int c = 0; c < N / 8; ++c)
        if (8 * c < rows) {
#pragma unroll
            for (int j = 8 * c; j < 8 * c + 8; ++j)
                if (j < rows) {
                    if (GATED && FP8) {
                        const float *m = s.amax + t0 + j;
                        const float scale = fp8_scale(fmaxf(fmaxf(m[0], m[GP_FEW]), fmaxf(m[2 * GP_FEW], m[3 * GP_FEW])));
                        if (there) static_cast<uint8_t *>(p.out)[at + (size_t)j * p.d_out] = (uint8_t)fp8_codes4(a[j], 0.f, 0.f, 0.f, scale);
                        if (place == 0) p.out_scales[(size_t)(r.row0 + t0 + j) * out_blocks + r.out0 / DIP_FP8_BLOCK] = scale;
                    } else if (there) {
                        if (!GATED && p.out_f32) static_cast<float *>(p.out)[at + (size_t)j * p.d_out] = a[j];
                        else static_cast<__nv_bfloat16 *>(p.out)[at + (size_t)j * p.d_out] = __float2bfloat16_rn(a[j]);
                    }
                }
        }
    if (GATED && FP8) out_barrier<K>();                 // (before the next tile's maxima)
}

// A piece of this warp's 32 rows leaves by way of shared memory: each thread brings PIECE bytes of its row, and the warp writes
// whole pieces row after row (a thread writing 16 bytes of its own row at a time touched 32 lines per instruction: 6000 cycles for
// a tile of 256 bfloat16 columns).  to: the piece of lane 0's row, `pitch` bytes from row to row; only rows below n, bytes below `bytes`.
template <class K>
__device__ __forceinline__ void leave(unsigned char *stage, const uint4 *v, char *to, size_t pitch, int n, int bytes)
{
    constexpr int Q = K::PIECE / 16, ROWS = 32 / Q, SHIFT = K::PIECE == 64 ? 1 : 2;       // 16-byte parts of a piece, rows per pass
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int q = 0; q < Q; ++q) *reinterpret_cast<uint4 *>(stage + lane * K::PIECE + ((q ^ (lane >> SHIFT & (Q - 1))) << 4)) = v[q];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < Q; ++i) {
        const int row = i * ROWS + lane / Q, q = lane % Q;
        const uint4 w = *reinterpret_cast<const uint4 *>(stage + row * K::PIECE + ((q ^ (row >> SHIFT & (Q - 1))) << 4));
        if (row < n && 16 * q < bytes) *reinterpret_cast<uint4 *>(to + row * pitch + 16 * q) = w;
    }
}

// The sums of any other tile: thread = row, values = its share of the columns, in two groups: H from the tile's output first on and H from
// second on (gate/up: gate, and the up of the same outputs).  row0, rows: this block's rows of the tile (may be none).
template <class K>
__device__ __forceinline__ void take_tile(const GroupedParams &p, GroupedSmem<K> &s, const Schedule<K> &plan, const Run &r, int row0, int rows,
                                          uint32_t lanes, int share, int row, int &n, int &groups)
{
    constexpr bool FP8 = K::FP8, GATED = K::GATED, PAIR = K::PAIR, SPLIT = K::SPLIT;
    constexpr int SHARES = K::OUT_WARPS / 4, C = GP_COLS / SHARES, H = C / 2;
    // the groups' columns; halves of a pair's accumulator have the first (second) half of both blocks' weights
    const int lane = threadIdx.x & 31;
    const int first = GATED || SPLIT ? H * share : C * share, second = GATED ? first : SPLIT ? GP_COLS / 2 + first : first + H;
    const int col0 = SPLIT ? C * share : first, col1 = GATED && !SPLIT ? GP_COLS / 2 + col0 : col0 + H;
    const int out_blocks = (p.d_out + DIP_FP8_BLOCK - 1) / DIP_FP8_BLOCK;
    float acc[C];
    if constexpr (FP8) {
#pragma unroll
        for (int j = 0; j < C; ++j) acc[j] = 0.f;
        // (which of the tile's two blocks of weights a group of columns belongs to)
        const bool block0 = !GATED && !SPLIT && share == 1, block1 = GATED || SPLIT || share == 1;
        // (registers: with 32 columns gate/up keeps some of its own in memory and a prompt's product of 5120 to 17920 takes 476 us instead
        // of 441; plain products keep 20 bytes a thread there (pairs; whole tiles 60), and take 675 instead of 701)
        constexpr int L = GATED ? 16 : 32;
        const uint32_t full = smem_u32(&s.sum_full[0][SPLIT ? share : 0]), empty = smem_u32(&s.sum_empty[0][SPLIT ? share : 0]);
        constexpr uint32_t NEXT = sizeof(s.sum_full[0]);             // from one accumulator's barrier to the other's
        for (int left = r.k1 - r.k0; left > 0; left -= GP_SCALE_STEPS, ++groups) {
            const int slot = groups % GP_SCALE_SLOTS;
            wait_on(smem_u32(&s.scale_full[slot]), (groups / GP_SCALE_SLOTS) & 1, s, p.status, p.wait_limit_ns);
            const float *xs = &s.row_scale[slot * GP_SCALE_STEPS][row];
            const float2 *ws = &s.w_scale[slot * GP_SCALE_STEPS];
            const int end = n + min(left, GP_SCALE_STEPS);
            for (; n < end; ++n, xs += GP_ROWS, ++ws) {
                const float x = *xs;
                const float2 w = *ws;
                const float s0 = x * (block0 ? w.y : w.x), s1 = x * (block1 ? w.y : w.x);
                const int buf = n & 1;
                wait_on(full + buf * NEXT, (n >> 1) & 1, s, p.status, p.wait_limit_ns);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                // one load is under way while the one in front is added (of L columns)
                const uint32_t from = lanes + buf * GP_COLS;
                uint32_t v[2][L];
                tmem_ld(from + col0, v[0]);
#pragma unroll
                for (int c = 0; c < C / L; ++c) {
                    tmem_wait(v[c & 1]);
                    if (c + 1 < C / L) {
                        tmem_ld(from + (L * (c + 1) < H ? col0 + L * (c + 1) : col1 + L * (c + 1) - H), v[(c + 1) & 1]);
                    } else {                         // all of it is in registers
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        arrive_first<PAIR>(empty + buf * NEXT, lane);
                    }
#pragma unroll
                    for (int j = 0; j < L; j += 2) fma2(acc[L * c + j], acc[L * c + j + 1], v[c & 1][j], v[c & 1][j + 1], L * c < H ? s0 : s1);
                }
            }
            __syncwarp();
            arrive_first<false>(smem_u32(&s.scale_empty[slot]), lane);
        }
    } else {
        const int buf = n & 1;
        wait_on(smem_u32(&s.sum_full[buf][0]), (n / 2) & 1, s, p.status, p.wait_limit_ns);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int c = 0; c < C / 16; ++c) {
            uint32_t v[16];
            tmem_ld(lanes + buf * GP_COLS + (16 * c < H ? col0 + 16 * c : col1 + 16 * c - H), v);
            tmem_wait(v);
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[16 * c + j] = __uint_as_float(v[j]);
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        arrive_first<PAIR>(smem_u32(&s.sum_empty[buf][0]), lane);
        ++n;
    }

    if (r.k1 - r.k0 < p.steps) {
        // parts are [share][column / 4][row][4]
        const size_t mine = (size_t)share * (C / 4) * GP_ROWS + row;
        float4 *to = reinterpret_cast<float4 *>(p.partials + plan.part_at(plan.block(), r.rest)) + mine;
        if (row < rows) {
#pragma unroll
            for (int j = 0; j < C / 4; ++j) to[j * GP_ROWS] = make_float4(acc[4 * j], acc[4 * j + 1], acc[4 * j + 2], acc[4 * j + 3]);
        }
        int b0, b1;
        if (!part_is_last(p, s, plan, r, b0, b1)) return;
#pragma unroll
        for (int j = 0; j < C; ++j) acc[j] = 0.f;
        if (row < rows) {
            for (int b = b0; b <= b1; ++b) {
                const float4 *from = reinterpret_cast<const float4 *>(p.partials + plan.part_at(b, r.rest)) + mine;
#pragma unroll
                for (int j = 0; j < C / 4; ++j) {
                    const float4 v = __ldcg(from + j * GP_ROWS);
                    acc[4 * j] += v.x;
                    acc[4 * j + 1] += v.y;
                    acc[4 * j + 2] += v.z;
                    acc[4 * j + 3] += v.w;
                }
            }
        }
    }

    const int warp_row = row & ~31, n_here = rows - warp_row;        // this warp's rows
    unsigned char *stage = s.out[(threadIdx.x >> 5) - 4];
    if (GATED) {
        const int o = r.out0 + first;
#pragma unroll
        for (int j = 0; j < H; ++j) acc[j] = silu_f32(acc[j]) * acc[H + j];
        if (FP8) {
            // a block of 128 outputs has a scale: two threads have a half each (widths are multiples of 32 outputs)
            float most = 0.f;
#pragma unroll
            for (int j = 0; j < H; ++j)
                if (o + (j & ~31) < p.d_out) most = fmaxf(most, fabsf(acc[j]));
            s.amax[share * GP_ROWS + row] = most;
            out_barrier<K>();
            const float scale = fp8_scale(fmaxf(most, s.amax[(share ^ 1) * GP_ROWS + row]));
            if (row < rows && share == 0) p.out_scales[(size_t)(row0 + row) * out_blocks + r.out0 / DIP_FP8_BLOCK] = scale;
            char *to = static_cast<char *>(p.out) + (size_t)(row0 + warp_row) * p.d_out + o;
            constexpr int B = K::PIECE;
#pragma unroll
            for (int c = 0; c < H / B; ++c) {
                uint4 v[B / 16];
#pragma unroll
                for (int q = 0; q < B / 16; ++q) {
                    const float *f = acc + c * B + 16 * q;
                    v[q] = make_uint4(fp8_codes4(f[0], f[1], f[2], f[3], scale), fp8_codes4(f[4], f[5], f[6], f[7], scale),
                                      fp8_codes4(f[8], f[9], f[10], f[11], scale), fp8_codes4(f[12], f[13], f[14], f[15], scale));
                }
                leave<K>(stage, v, to + c * B, p.d_out, n_here, p.d_out - o - c * B);
            }
            out_barrier<K>();                      // (before the next tile's maxima)
            return;
        }
    }
    const int item = !GATED && p.out_f32 ? 4 : 2;
    const size_t pitch = (size_t)p.d_out * item;
    char *to = static_cast<char *>(p.out) + ((size_t)(row0 + warp_row) * p.d_out + r.out0) * item;
    constexpr int B = K::PIECE;
#pragma unroll
    for (int g = 0; g < (GATED ? 1 : 2); ++g) {
        const int o = g ? second : first, left = (p.d_out - r.out0 - o) * item;
        if (item == 4) {
#pragma unroll
            for (int c = 0; c < 4 * H / B; ++c) {
                uint4 v[B / 16];
#pragma unroll
                for (int q = 0; q < B / 16; ++q) {
                    const float *f = acc + g * H + c * (B / 4) + 4 * q;
                    v[q] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
                }
                leave<K>(stage, v, to + o * 4 + c * B, pitch, n_here, left - c * B);
            }
        } else {
#pragma unroll
            for (int c = 0; c < 2 * H / B; ++c) {
                uint4 v[B / 16];
#pragma unroll
                for (int q = 0; q < B / 16; ++q) v[q] = bf16x8(acc + g * H + c * (B / 2) + 8 * q);
                leave<K>(stage, v, to + o * 2 + c * B, pitch, n_here, left - c * B);
            }
        }
    }
}

// Every warp's roles are through (PAIR: in both blocks: the first one's MMAs have read the second one's memory, all has arrived at its
// barriers), and each block knows of the other's failure.
template <bool PAIR, int THREADS, typename Smem>
__device__ __forceinline__ void roles_end(Smem &s, int tid)
{
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    asm volatile("barrier.cta.sync 3, %0;" ::"n"(THREADS) : "memory");
    if (PAIR) {
        if (tid == 0 && *(volatile int *)&s.fail) peer_store(&s.peer_fail, 1);
        __syncwarp();
        pair_barrier();
    }
}
template <bool PAIR, typename Smem>
__device__ __forceinline__ bool gave_up(Smem &s) { return (*(volatile int *)&s.fail | (PAIR ? *(volatile int *)&s.peer_fail : 0)) != 0; }

template <class K>
__global__ void __launch_bounds__(K::THREADS, 1)
grouped_kernel(const __grid_constant__ CUtensorMap rows_map, const __grid_constant__ CUtensorMap w_map,
               const __grid_constant__ CUtensorMap w2_map, const GroupedParams p)
{
    constexpr bool FP8 = K::FP8, GATED = K::GATED, PAIR = K::PAIR, FEW = K::FEW, SPLIT = K::SPLIT;
    extern __shared__ unsigned char gp_smem_raw[];
    using Smem = GroupedSmem<K>;
    Smem &s = *reinterpret_cast<Smem *>((reinterpret_cast<uintptr_t>(gp_smem_raw) + 1023) & ~(uintptr_t)1023);
    constexpr int STAGES = K::STAGES, PER_STEP = FP8 ? GP_STEP_BYTES : GP_STEP_BYTES / 2;
    DIP_TRACE_MIN(p.tr, 0);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = PAIR ? blockIdx.x & 1 : 0;      // (clusters are two neighbouring blocks)

    if (warp == 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem_base)),
                         "n"(GP_TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem_base)),
                         "n"(GP_TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    if (tid == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(&s.full[i], 1);
            mbar_init(&s.empty[i], SPLIT ? 2 : 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&s.sum_full[i >> 1][i & 1], 1);
            mbar_init(&s.sum_empty[i >> 1][i & 1], (PAIR ? 2 : 1) * K::OUT_WARPS / (SPLIT ? 2 : 1));
        }
        for (int i = 0; i < GP_SCALE_SLOTS; ++i) {
            mbar_init(&s.scale_full[i], 32);
            mbar_init(&s.scale_empty[i], K::OUT_WARPS);
        }
        mbar_init(&s.drained[0], 1);
        mbar_init(&s.drained[1], 1);
        s.fail = s.peer_fail = s.issued = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&rows_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&w_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&w2_map) : "memory");
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // rows and offsets come from the kernels in front; weights do too, as far as the library can know, so before they are through it only
    // asks L2 for the first ones, where there are no offsets to wait for
    const Schedule<K> plan = {p, s.plan};
    if (warp != 0 || p.offset) dip_grid_dependency_wait();
    DIP_TRACE_MIN(p.tr, 1);
    if (warp == 0) {
        __syncwarp();
        grouped_plan(p, plan.ROWS, s.plan);
        __syncwarp();
        if (lane == 0) plan.divide();
        __syncwarp();
        if (!p.offset) {
            Run r;
            if (FEW && plan.get(0, r) && elect_one()) {
                for (int k = r.k0; k < min(r.k0 + STAGES, r.k1); ++k) {
                    tma_prefetch(&w_map, k * PER_STEP, r.out0);
                    tma_prefetch(GATED ? &w2_map : &w_map, k * PER_STEP, GATED ? r.out0 : r.out0 + GP_COLS / 2);
                }
            }
            __syncwarp();
            dip_grid_dependency_wait();
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (PAIR) {
        __syncthreads();
        pair_barrier();                              // (the other block's barriers are set up)
    } else if (warp == 0) {                          // (goes on to its copies)
        asm volatile("barrier.cta.arrive 2, %0;" ::"n"(K::THREADS) : "memory");
    } else {
        asm volatile("barrier.cta.sync 2, %0;" ::"n"(K::THREADS) : "memory");
    }
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    dip_launch_dependents();
    const uint32_t tmem = s.tmem_base;               // (warp 0 has no use for it)
    bool failed = false;

    if (warp < 4) {
        if (!FEW) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(K::REGS_FEW));
        if (warp == 0) {
            Run r;
            int g = 0;                               // steps so far
            for (int i = 0; !failed && plan.get(i, r); ++i) {
                const bool both = r.rows > GP_BOX;               // (few)
                const int w_row = r.expert * p.d_out + r.out0, row0 = r.row0 + rank * GP_ROWS;
                // (plain: the tile's second half may lie behind the last output; PAIR: the second block may have no rows)
                const bool second = GATED || r.out0 + GP_COLS / 2 < p.d_out, some = rank * GP_ROWS < r.rows;
                const unsigned bytes = PAIR ? GP_B_BYTES + (r.rows > GP_ROWS ? 2 : 1) * GP_A_BYTES
                                            : (FEW ? (both ? 2 : 1) * GP_BOX * GP_STEP_BYTES : GP_A_BYTES) + (second ? GP_B_BYTES : GP_B_BYTES / 2);
                int x = r.k0 * PER_STEP;
                for (int k = r.k0; k < r.k1; ++k, ++g, x += PER_STEP) {
                    const int st = g % STAGES;
                    if (g >= STAGES && !warp_wait(&s.empty[st], (g / STAGES - 1) & 1, p.wait_limit_ns)) {
                        failed = true;
                        break;
                    }
                    if (elect_one()) {
                        if (rank == 0) mbar_expect_tx(&s.full[st], bytes);
                        if (PAIR) {
                            if (GATED) tma_load<PAIR>(s.b[st], rank ? &w2_map : &w_map, x, w_row, &s.full[st]);
                            else tma_load<PAIR>(s.b[st], &w_map, x, w_row + rank * (GP_COLS / 2), &s.full[st]);
                            if (some) tma_load<PAIR>(s.a[st], &rows_map, x, row0, &s.full[st]);
                        } else {
                            if (GATED) {
                                tma_load<PAIR>(s.b[st], &w_map, x, w_row, &s.full[st]);
                                tma_load<PAIR>(s.b[st] + GP_B_BYTES / 2, &w2_map, x, w_row, &s.full[st]);
                            } else {
                                tma_load<PAIR>(s.b[st], second ? &w2_map : &w_map, x, w_row, &s.full[st]);
                            }
                            tma_load<PAIR>(s.a[st], &rows_map, x, r.row0, &s.full[st]);
                            if (FEW && both) tma_load<PAIR>(s.a[st] + GP_BOX * GP_STEP_BYTES, &rows_map, x, r.row0 + GP_BOX, &s.full[st]);
                        }
                    }
                    __syncwarp();
                }
            }
            if (lane == 0) s.issued = g;
        } else if (Smem::RING && warp == 3) {
            // four rows a lane; the first lanes the weights' scales
            const int out_blocks = (p.d_out + DIP_FP8_BLOCK - 1) / DIP_FP8_BLOCK;
            Run r;
            int g = 0;                               // groups so far
            for (int i = 0; !failed && plan.get(i, r); ++i) {
                const int last_row = r.row0 + r.rows - 1, ob = r.out0 / DIP_FP8_BLOCK + (GATED ? 0 : lane & 1);
                const float *x[4];
#pragma unroll
                for (int m = 0; m < 4; ++m) x[m] = p.row_scales + (size_t)min(r.row0 + rank * GP_ROWS + 32 * m + lane, last_row) * p.steps;
                const float *ws = (GATED && (lane & 1) ? p.up_scales : p.w_scales) + ((size_t)r.expert * out_blocks + min(ob, out_blocks - 1)) * p.steps;
                for (int k0 = r.k0; k0 < r.k1; k0 += GP_SCALE_STEPS, ++g) {
                    const int slot = g % GP_SCALE_SLOTS;
                    if (g >= GP_SCALE_SLOTS && !warp_wait(&s.scale_empty[slot], (g / GP_SCALE_SLOTS - 1) & 1, p.wait_limit_ns)) {
                        failed = true;
                        break;
                    }
#pragma unroll
                    for (int q = 0; q < GP_SCALE_STEPS; ++q) {
                        const int k = min(k0 + q, r.k1 - 1);
#pragma unroll
                        for (int m = 0; m < 4; ++m) copy4(&s.row_scale[slot * GP_SCALE_STEPS + q][32 * m + lane], x[m] + k);
                    }
                    if (lane < 2 * GP_SCALE_STEPS)
                        copy4(reinterpret_cast<float *>(s.w_scale) + slot * 2 * GP_SCALE_STEPS + lane, ws + min(k0 + (lane >> 1), r.k1 - 1));
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&s.scale_full[slot])) : "memory");
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        } else if ((warp == 1 || (SPLIT && warp == 2)) && rank == 0) {
            const int half = warp - 1;
            Run r;
            int g = 0, n = 0;                        // steps, accumulators so far
            for (int i = 0; !failed && plan.get(i, r); ++i) {
                const uint32_t shape = grouped_shape<FP8, PAIR>(FEW ? (r.rows + 15) / 16 * 16 : SPLIT ? GP_COLS / 2 : GP_COLS);
                for (int k = r.k0; k < r.k1; ++k, ++g) {
                    const int st = g % STAGES, buf = n & 1;
                    const bool first = FP8 || k == r.k0, last = FP8 || k == r.k1 - 1;
                    if ((first && n >= 2 && !warp_wait(&s.sum_empty[buf][half], (n / 2 - 1) & 1, p.wait_limit_ns)) ||
                        !warp_wait(&s.full[st], (g / STAGES) & 1, p.copy_wait_ns)) {
                        failed = true;
                        break;
                    }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    // a half of N = 128 is 64 rows of each block's weights
                    const uint64_t a = operand_desc(s.a[st]), b = operand_desc(s.b[st]) + (SPLIT ? half * (64 * GP_STEP_BYTES >> 4) : 0);
                    const uint32_t to = tmem + buf * GP_COLS + (SPLIT ? half * (GP_COLS / 2) : 0);
                    if (elect_one()) {
                        if (!FEW) {
#pragma unroll
                            for (int q = 0; q < 4; ++q)          // 32 bytes of K each
                                grouped_mma<FP8, PAIR>(to, a + 2 * q, b + 2 * q, shape, (first && q == 0) ? 0u : 1u);
                        } else {
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                grouped_mma<FP8, PAIR>(to, b + 2 * q, a + 2 * q, shape, (first && q == 0) ? 0u : 1u);
                                grouped_mma<FP8, PAIR>(to + GP_COLS / 2, b + (GP_B_BYTES / 2 >> 4) + 2 * q, a + 2 * q, shape,
                                                       (first && q == 0) ? 0u : 1u);
                            }
                        }
                        grouped_commit<PAIR>(&s.empty[st]);
                        if (last) grouped_commit<PAIR>(&s.sum_full[buf][half]);
                    }
                    __syncwarp();
                    if (last) ++n;
                }
            }
        }
        if (failed) {
            *(volatile int *)&s.fail = 1;
            atomicExch(p.status, 1);
        }
        // All roles are through.  Where any wait has run out, whoever's it was, MMAs and copies may still be under way (the last
        // steps' copies, though the warp that issued them knows of nothing): they are waited for.
        roles_end<PAIR, K::THREADS>(s, tid);
        if (gave_up<PAIR>(s)) {
            if (warp == 1 || (SPLIT && warp == 2)) {
                if (rank == 0 && elect_one()) grouped_commit<PAIR>(&s.drained[warp - 1]);
                __syncwarp();
                warp_wait(&s.drained[warp - 1], 0, p.wait_limit_ns);
            }
            if (warp == 0 && rank == 0) {
                const auto second_bytes = [&](int j) {
                    Run r = {};
                    for (int i = 0, step = 0; plan.get(i, r) && step + r.k1 - r.k0 <= j; ++i) step += r.k1 - r.k0;
                    return (unsigned)(K::B_BYTES + (r.rows > GP_ROWS ? K::A_BYTES : 0));
                };
                drain_copies<STAGES, PAIR>(s.full, s.issued, PAIR ? peer_load(&s.issued) : 0, second_bytes, p.wait_limit_ns);
            }
        }
    } else {
        if (!FEW) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(K::REGS_MANY));
        const int share = (warp - 4) >> 2, place = (warp & 3) * 32 + lane;     // lane of tensor memory
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        int n = 0, groups = 0;                       // accumulators, groups of scales so far
        Run r;
        for (int i = 0; plan.get(i, r); ++i) {
            if constexpr (FEW) take_few<K>(p, s, plan, r, lanes, share, place, n);
            else take_tile<K>(p, s, plan, r, r.row0 + rank * GP_ROWS, min(GP_ROWS, r.rows - rank * GP_ROWS), lanes, share, place, n, groups);
        }
        roles_end<PAIR, K::THREADS>(s, tid);
    }
    if (PAIR && gave_up<PAIR>(s)) pair_barrier();       // (neither leaves before the first one has waited for all)
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 1) {
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(GP_TMEM_COLS) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(GP_TMEM_COLS) : "memory");
    }
    DIP_TRACE_MAX(p.tr, 2);
}

// Self-test of a wait that runs out: warp 1 of block `failing` waits for what never comes, warp 2 for what warp 1 would have done, and warp 0 of
// the first block then waits for the copies that `mine` and `other` steps have on their way, as in grouped_kernel.  No copy is: warp 3 stands
// for them, and counts their bytes off late.  report: how many came; how many had when the drain was through.
template <bool PAIR>
__global__ void __launch_bounds__(128, 1)
group_waits_selftest_kernel(int mine, int other, int failing, int *status, unsigned long long limit_ns, unsigned long long bound_ns,
                            unsigned long long *report)
{
    constexpr int STAGES = 5;
    constexpr unsigned FIRST = 1024, SECOND = 512;   // bytes of a step, the second block's of them
    struct Smem {
        uint64_t full[STAGES], never, sum_full;
        int fail, peer_fail, issued;
    };
    __shared__ Smem s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = PAIR ? blockIdx.x & 1 : 0;
    const int landed = max(0, (PAIR ? max(mine, other) : mine) - STAGES);      // steps that are through
    if (tid == 0) {
        for (int i = 0; i < STAGES; ++i) mbar_init(&s.full[i], 1);
        mbar_init(&s.never, 1);
        mbar_init(&s.sum_full, 1);
        s.fail = s.peer_fail = 0;
        s.issued = rank ? other : mine;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int j = 0; rank == 0 && j < mine; ++j) {
            mbar_expect_tx(&s.full[j % STAGES], FIRST + (PAIR ? SECOND : 0));
            if (j < landed) mbar_complete_tx(&s.full[j % STAGES], FIRST + (PAIR ? SECOND : 0));
        }
    }
    __syncthreads();
    if (PAIR) pair_barrier();
    if (warp == 3) {
        if (PAIR) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // (holds nobody up)
        const unsigned long long t0 = dip_gtime();
        for (int i = 0; i < (1 << 22) && dip_gtime() - t0 < limit_ns + min(limit_ns, 100000000ull); ++i) __nanosleep(500);
        if (lane == 0) {
            for (int j = landed; j < s.issued; ++j) {
                atomicAdd(report, 1ull);
                __threadfence();
                if (rank == 0) mbar_complete_tx(&s.full[j % STAGES], FIRST);
                else asm volatile("mbarrier.complete_tx.relaxed.cluster.shared::cluster.b64 [%0], %1;" ::"r"(peer_word(&s.full[j % STAGES])), "r"(SECOND)
                                  : "memory");
            }
        }
        __syncwarp();
        if (PAIR) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        bool failed = false;
        if (rank == failing) {
            if (warp == 1) failed = !warp_wait(&s.never, 0, limit_ns);
            if (warp == 2) wait_on(smem_u32(&s.sum_full), 0, s, status, bound_ns);
        }
        if (failed) {
            *(volatile int *)&s.fail = 1;
            atomicExch(status, 1);
        }
        roles_end<PAIR, 96>(s, tid);
        if (gave_up<PAIR>(s) && warp == 0 && rank == 0) {
            drain_copies<STAGES, PAIR>(s.full, s.issued, PAIR ? peer_load(&s.issued) : 0, [](int) { return SECOND; }, bound_ns);
            if (lane == 0) report[1] = atomicAdd(report, 0ull);
        }
    }
    if (PAIR && gave_up<PAIR>(s)) pair_barrier();
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The CUDA driver's encoder, looked up once (the library does not link against libcuda).
EncodeTiled encoder()
{
    static const EncodeTiled fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return (EncodeTiled)f;
    }();
    return fn;
}

// Pieces of `box` rows by 128 bytes of a row-major [n][d] matrix, laid down with the 128-byte swizzle; zeros outside.
bool encode(CUtensorMap *map, const void *p, bool fp8, size_t n, int d, int box)
{
    const int item = fp8 ? 1 : 2;
    const cuuint64_t dims[2] = {(cuuint64_t)d, (cuuint64_t)n}, strides[1] = {(cuuint64_t)d * item};
    const cuuint32_t piece[2] = {(cuuint32_t)(GP_STEP_BYTES / item), (cuuint32_t)box}, one[2] = {1, 1};
    return encoder()(map, fp8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(p), dims, strides,
                     piece, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class K>
cudaError_t launch(dip_ctx *ctx, int ctas, cudaStream_t stream, const CUtensorMap (&m)[3], const GroupedParams &p)
{
    static dip_per_device_once once;
    const auto kernel = grouped_kernel<K>;
    const size_t smem = sizeof(GroupedSmem<K>) + 1024;
    static_assert(sizeof(GroupedSmem<K>) + 1024 <= 227 * 1024, "fits a CTA's shared memory");
    // (the warps that take sums out would wait for ever for registers that the launch does not have)
    static const bool enough = [&] {
        cudaFuncAttributes a;
        return K::FEW || (cudaFuncGetAttributes(&a, kernel) == cudaSuccess &&
                          a.numRegs * (4 + K::OUT_WARPS) >= K::REGS_FEW * 4 + K::REGS_MANY * K::OUT_WARPS);
    }();
    if (!enough) return cudaErrorLaunchOutOfResources;
    const cudaError_t e = dip_raise_smem_limit(once, ctx->device, kernel, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(K::THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = K::PAIR ? 2 : 1;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, m[0], m[1], m[2], p);
}

template <bool FP8, bool GATED>
cudaError_t launch(int mode, dip_ctx *ctx, int ctas, cudaStream_t stream, const CUtensorMap (&m)[3], const GroupedParams &p)
{
    return mode == GP_PAIR    ? launch<Kind<FP8, GATED, GP_PAIR>>(ctx, ctas, stream, m, p)
           : mode == GP_WHOLE ? launch<Kind<FP8, GATED, GP_WHOLE>>(ctx, ctas, stream, m, p)
                              : launch<Kind<FP8, GATED, GP_FEW_ROWS>>(ctx, ctas, stream, m, p);
}

}  // namespace

// Few up to, and pairs from this many rows per expert on (the average over as many experts as can have any).  In us, few / whole tiles:
// 8 rows for each of 32 experts, 1024 to 1024, 18.8 / 19.3 (8-bit 10.2 / 11.5), 32 rows 20.3 / 19.8 (12.9 / 11.7); one expert, 4096 to 5120, 8 rows
// 18.3 / 26.9 (16.2 / 22.0), 24 rows 29.0 / 25.6 (24.8 / 22.8).  Whole tiles / pairs: 100 rows for each of 64 experts, gate/up of 2048 to 1408, 139 / 164;
// 16 experts, 4096 to 4096, 150 rows 116 / 123, 200 rows 149 / 145; 1024 rows for each of 8, gate/up of 4096 to 14336, 1648 / 1430 (8-bit
// 1304 / 1255).  What this leaves out: 8-bit pairs were compared at 1024 rows only, and groups of unequal size not at all (an expert of 257 to
// 384 rows fills half of its second pair tile, or less).
constexpr int GP_FEW_UP_TO = 12, GP_PAIR_ROWS = 192;

dip_status dip_launch_grouped(dip_ctx *ctx, const dip_grouped_matrix &w, const dip_grouped_matrix *up, const void *rows,
                              const float *row_scales, int n_rows, const int32_t *offset, void *out, bool out_f32, float *out_scales,
                              cudaStream_t stream)
{
    const bool fp8 = w.wtype == DIP_W_FP8_B128;
    const int met = min(w.n_experts, n_rows);
    const int mode = n_rows <= GP_FEW_UP_TO * met ? GP_FEW_ROWS : n_rows >= GP_PAIR_ROWS * met && ctx->sm_count % 2 == 0 ? GP_PAIR : GP_WHOLE;
    const size_t w_rows = (size_t)w.n_experts * w.d_out;
    // the rows; half of a tile's weights; the other half (gate/up), or both at once
    CUtensorMap maps[3];
    if (!encoder() || !encode(&maps[0], rows, fp8, n_rows, w.d_in, mode == GP_FEW_ROWS ? GP_BOX : GP_ROWS) ||
        !encode(&maps[1], w.values, fp8, w_rows, w.d_in, GP_COLS / 2) ||
        !encode(&maps[2], up ? up->values : w.values, fp8, w_rows, w.d_in, up ? GP_COLS / 2 : GP_COLS)) {
        snprintf(ctx->err, sizeof(ctx->err), "cuTensorMapEncodeTiled failed");
        return DIP_ERR_CUDA;
    }
    const int width = up ? GP_COLS / 2 : GP_COLS, tile_rows = mode == GP_PAIR ? 2 * GP_ROWS : mode == GP_WHOLE ? GP_ROWS : GP_FEW;
    GroupedParams p = {};
    p.w_scales = w.scales;
    p.up_scales = up ? up->scales : nullptr;
    p.row_scales = row_scales;
    p.n_experts = w.n_experts;
    p.d_out = w.d_out;
    p.d_in = w.d_in;
    p.n_rows = n_rows;
    p.steps = (w.d_in * (fp8 ? 1 : 2) + GP_STEP_BYTES - 1) / GP_STEP_BYTES;
    p.n_cols = (w.d_out + width - 1) / width;
    p.join = mode == GP_FEW_ROWS ? GP_JOIN_FEW + n_rows / met : GP_JOIN;
    p.offset = offset;
    p.out = out;
    p.out_scales = out_scales;
    p.out_f32 = out_f32;
    p.partials = ctx->partials;
    p.tickets = ctx->group_tickets;
    p.status = ctx->status;
    p.copy_wait_ns = ctx->wait_limit_ns;
    p.wait_limit_ns = ctx->block_wait_ns;
    p.tr = dip_trace_slot(ctx, up ? 10 : 11);
    // no more blocks than there can be parts
    const long long tiles = (long long)((n_rows + tile_rows - 1) / tile_rows + met - 1) * p.n_cols;
    const long long most = max(tiles, tiles * p.steps / GP_MIN_STEPS);
    const int ctas = mode == GP_PAIR ? 2 * (int)min((long long)ctx->sm_count / 2, most) : (int)min((long long)ctx->sm_count, most);
    const auto start = fp8 ? (up ? launch<true, true> : launch<true, false>) : (up ? launch<false, true> : launch<false, false>);
    DIP_CUDA_TRY(ctx, start(mode, ctx, ctas, stream, maps, p));
    return DIP_OK;
}

dip_status dip_launch_group_waits_selftest(dip_ctx *ctx, unsigned long long limit_ns, unsigned long long *report, cudaStream_t stream)
{
    // steps that each block has asked for, and which one's wait runs out; the first two are blocks by themselves
    static const int cases[DIP_SELFTEST_GROUP_CASES][3] = {{3, 0, 0}, {12, 0, 0}, {4, 4, 0}, {13, 13, 1}, {9, 5, 0}, {9, 6, 1}, {5, 9, 0}, {2, 4, 1}};
    DIP_CUDA_TRY(ctx, cudaMemsetAsync(report, 0, 2 * DIP_SELFTEST_GROUP_CASES * sizeof(*report), stream));
    for (int i = 0; i < DIP_SELFTEST_GROUP_CASES; ++i) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(i < 2 ? 1 : 2);
        cfg.blockDim = dim3(128);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = cfg.gridDim.x;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        DIP_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, i < 2 ? group_waits_selftest_kernel<false> : group_waits_selftest_kernel<true>, cases[i][0],
                                             cases[i][1], cases[i][2], ctx->status, limit_ns, ctx->block_wait_ns, report + 2 * i));
    }
    return DIP_OK;
}
