// What the kernels of grouped products share: waits, copies, tensor memory, and the schedule by which tiles are dealt out to blocks.
#pragma once

#include <cuda.h>

#include "common.cuh"
#include "gemv_common.cuh"

namespace {

constexpr int GP_ROWS = DIP_GROUP_ROWS, GP_COLS = DIP_GROUP_COLS;
constexpr int GP_STEP_BYTES = 128;                  // of a row, per step
constexpr int GP_TMEM_COLS = 512;
constexpr int GP_MIN_STEPS = 4;                     // a part of a tile has at least so many
constexpr int GP_TWO_RUNS = 6;                      // steps' worth of time that a block loses between two runs
constexpr int GP_CHUNK = 12;                        // row tiles that go through an expert's weights together

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
// (32 bits hold it all: fewer than 2^24 tiles, and fewer cut ones than blocks, of at most 512 steps, whose number is multiplied by that of blocks.)
static_assert((long long)(DIP_MAX_TOKENS * DIP_MAX_TOP_K / GP_ROWS + DIP_MAX_EXPERTS) * (DIP_MAX_OUT / GP_COLS) < 1 << 24, "tiles of 128 rows by 256 outputs");
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
template <class K, class Smem>
__device__ __forceinline__ bool part_is_last(const GroupedParams &p, Smem &s, const Schedule<K> &plan, const Run &r, int &b0, int &b1)
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

}  // namespace
