// Products of groups of few rows with 4-bit weights: y[r] = W[e(r)] rows[r], h[r] = silu(Wg[e(r)] rows[r]) * (Wu[e(r)] rows[r]), where
// W[o][i] = (code - 8) * S[i / 128][o].  Per group of 128 input indices the products code * x are exact in binary32 and are summed by the
// tensor cores (m16n8k16: 16 outputs x 16 inputs x 8 rows of bfloat16); each group's sum is then multiplied by its scale into the output's
// binary32 sum.  Nothing but y is rounded to fewer bits.
//
// Bound by the stream of codes, so what matters is that every SM has enough of it under way and that the ALUs, which turn codes into
// bfloat16, keep up:
//   * A unit is 64 outputs (gate/up: 32 of each) by one group: 4 KB of codes, 64 bytes of a row at a time.  Each warp has a ring of
//     units that it fills with asynchronous copies of its own and waits for by itself; a lane reads back what it copied.  (Twelve warps, or eight of
//     more registers for 9 rows and more: with twelve 16 rows of 4096 to 102400 took 105 us instead of 77.)
//   * A lane's 16 bytes of a row are 32 consecutive codes, and the sums of a group do not depend on the order of its inputs, so the four lanes
//     of a quad simply take a quarter of the group each, and an MMA takes the codes that one AND brings out of a word, nibbles s and s + 4
//     (int4_codes.cuh).  x is paired alike.
//   * All units, tile after tile, are dealt out to the blocks in equal runs, and a block's to its warps: whatever the sizes, nobody has
//     more than a unit too many.  Where whole tiles are hardly worse for the blocks, they stay whole: parts of a tile that meet in
//     the workspace cost a write, a count and a read (the block that comes last adds them up in order; nobody waits).
// One row of 4096 to 102400 takes 50 us (4.3 TB/s; 218 MB at the measured rate are 33): its copies alone take 42, since they come as runs of 64 bytes of
// a row (longer runs reach more: pieces of 512 bytes 6.3 TB/s), the rest without them 44.  Codes to bfloat16 are 288 of some 570 instructions of a unit; the
// other half are copies and their addresses, reads of shared memory, MMAs, x, scales and sums (ALU pipe busy 48 %, multiply-adds 44, issue slots 58, mma.sync 26).  Twelve
// warps or eight, four MMAs side by side or one, bare codes with the 8 taken off the sums (46 us for one row, 53 instead of 50 for eight) change little.
// Before and behind it 5 us go into the first loads and the last sums.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "float8.cuh"
#include "gemv_common.cuh"
#include "int4_codes.cuh"

namespace {

template <int NT> constexpr int IF_WARPS = NT == 1 ? 12 : 8;
template <int NT> constexpr int IF_THREADS = IF_WARPS<NT> * 32;
constexpr int IF_OUTS = 64;                 // outputs of a tile (gate/up: as many sums, of half as many outputs)
constexpr int IF_PITCH = IF_OUTS + 4;       // floats of a row of partial sums in shared memory (conflict-free)
constexpr int IF_STAGES = 3;                // units of a warp that are under way or in hand
// Units' worth of time that parts of a tile take to meet.  (us, whole tiles / cut ones: one row of 5120 to 17920, 80 units a block or 75.7, 18.2 / 21.4;
// 4096 to 4096 8.8 / 10.7; 17920 to 5120, 140 or 75.7, 23.6 / 21.1.)
constexpr int IF_JOIN = 24;

struct FewParams {
    const uint8_t *codes, *up_codes;
    const __half *scales, *up_scales;
    const __nv_bfloat16 *rows;
    const int32_t *offset;
    int n_experts, d_out, d_in, n_rows, groups, n_cols;
    void *out;
    int out_f32;
    float *partials;
    unsigned int *tickets;
    unsigned long long *tr;
};

struct __align__(16) FewStage {
    uint4 codes[8][32];                     // tile of 16 outputs, half of it; lane
    __half scales[IF_OUTS];
};

// A tile: 8 * NT rows of one expert, 64 sums of each.
struct FewTile {
    int expert, row0, rows, out0;
    int w0, w1;                             // the warps that have units of it
    int b0, b1;                             // and the blocks (b0 == b1: this one alone)
};

template <int NT> struct __align__(16) FewSmem {
    static constexpr int TILES = NT == 1 ? 20 : 4;      // that a block has in hand at a time (what there is room for)
    FewStage ring[IF_WARPS<NT>][IF_STAGES];
    float part[IF_WARPS<NT> + TILES][8 * NT][IF_PITCH];
    FewTile tile[TILES];
    int start[DIP_MAX_EXPERTS + 1];         // first row of each expert
    int tiles[DIP_MAX_EXPERTS + 1];         // tiles in front of it
    int last;
};

// 16 bytes to shared memory, asynchronously; or zeros.
__device__ __forceinline__ void copy16(void *dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16_or_0(void *dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// The same values, times one: for the order in which the compiler then puts a unit's instructions.  (8 rows of 4096 to 102400, us among passes with
// changing inputs: 56.3 with it, 57.9 without, 58.6 with an empty statement in its place.)
__device__ __forceinline__ uint32_t placed(uint32_t x)
{
    uint32_t v;
    asm volatile("mul.rn.bf16x2 %0, %1, %2;" : "=r"(v) : "r"(x), "r"(0x3f803f80u));
    return v;
}

// First rows and tiles of the experts, by one warp.
template <int NT>
__device__ __forceinline__ void few_plan(const FewParams &p, FewSmem<NT> &s)
{
    const int lane = threadIdx.x & 31, each = (p.n_experts + 32) / 32;
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
        if (i < p.n_experts) n += (s.start[i + 1] - s.start[i] + 8 * NT - 1) / (8 * NT) * p.n_cols;
    }
    int incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    for (int i = i0; i < i1; ++i) s.tiles[i] += incl - n;
}

// Of n units dealt out to `parts` in runs that differ by one at most: where run i starts, and whose a unit is (no run is empty: parts <= n).
__device__ __forceinline__ int run_start(int n, int parts, int i)
{
    const int each = n / parts;
    return each * i + min(i, n - each * parts);
}
__device__ __forceinline__ int run_of(int n, int parts, int unit)
{
    const int each = n / parts, longer = n - each * parts, of_these = longer * (each + 1);
    return unit < of_these ? unit / (each + 1) : longer + (unit - of_these) / each;
}

// (32 bits hold all numbers of units: a call of more goes to the kernel for many rows)
template <bool GATED, int NT>
__global__ void __launch_bounds__(IF_THREADS<NT>, 1)
int4_few_kernel(const FewParams p)
{
    extern __shared__ unsigned char if_smem_raw[];
    using Smem = FewSmem<NT>;
    Smem &s = *reinterpret_cast<Smem *>(if_smem_raw);
    constexpr int STAGES = IF_STAGES, FULL = GATED ? IF_OUTS / 16 : IF_OUTS / 8;      // eights of outputs of a whole tile
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane >> 2, in_quad = lane & 3;
    DIP_TRACE_MIN(p.tr, 0);
    dip_grid_dependency_wait();
    DIP_TRACE_MIN(p.tr, 1);
    if (warp == 0) few_plan(p, s);
    __syncthreads();
    dip_launch_dependents();

    const int tiles = s.tiles[p.n_experts], G = p.groups, blocks = gridDim.x, units = tiles * G;
    const bool whole = (tiles + blocks - 1) / blocks * G <= units / blocks + IF_JOIN;
    const int parts = min(blocks, whole ? tiles : units);
    int u0 = 0, u1 = 0;                     // this block's units
    if ((int)blockIdx.x < parts) {
        u0 = whole ? run_start(tiles, parts, blockIdx.x) * G : run_start(units, parts, blockIdx.x);
        u1 = whole ? run_start(tiles, parts, blockIdx.x + 1) * G : run_start(units, parts, blockIdx.x + 1);
    }

    while (u0 < u1) {
        // the next tiles
        const int t0 = u0 / G, t1 = min(t0 + Smem::TILES, (u1 + G - 1) / G), end = min(u1, t1 * G), n = end - u0, warps = min(IF_WARPS<NT>, n);
        if (tid < t1 - t0) {
            const int tile = t0 + tid;
            int lo = 0, hi = p.n_experts;   // the expert with tiles[e] <= tile < tiles[e + 1]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s.tiles[mid] <= tile) lo = mid;
                else hi = mid;
            }
            const int rows = s.start[lo + 1] - s.start[lo], chunks = (rows + 8 * NT - 1) / (8 * NT), in = tile - s.tiles[lo], col = in / chunks;
            const int first = (in - col * chunks) * 8 * NT, a = max(tile * G, u0), z = min((tile + 1) * G, end);
            FewTile t = {lo, s.start[lo] + first, min(8 * NT, rows - first), col * (GATED ? IF_OUTS / 2 : IF_OUTS)};
            t.w0 = run_of(n, warps, a - u0);
            t.w1 = run_of(n, warps, z - 1 - u0);
            t.b0 = t.b1 = blockIdx.x;
            if (z - a < G) {
                t.b0 = run_of(units, parts, tile * G);
                t.b1 = run_of(units, parts, (tile + 1) * G - 1);
            }
            s.tile[tid] = t;
        }
        __syncthreads();
        if (warp < warps) {
            const int first = run_start(n, warps, warp), stop = run_start(n, warps, warp + 1);
            // what is copied next: unit, its tile (among those in hand) and group
            int load = first, lt = (u0 + first) / G - t0, lg = u0 + first - (lt + t0) * G;
            const size_t half = (size_t)p.d_in / 2;
            const uint8_t *from_codes, *from_up = nullptr;                  // of this lane's row of the first 8 outputs
            const __half *from_scales;
            int eights;                                                     // eights of the tile's outputs that there are
            const auto locate = [&] {
                const FewTile &t = s.tile[lt];
                const size_t o = (size_t)t.expert * p.d_out + t.out0;
                from_codes = p.codes + (o + quad) * half + in_quad * 16;
                if (GATED) from_up = p.up_codes + (o + quad) * half + in_quad * 16;
                from_scales = (GATED && (lane & 4) ? p.up_scales : p.scales) + (size_t)t.expert * p.groups * p.d_out + t.out0 + lane % FULL * 8;
                eights = min(FULL, (p.d_out - t.out0) / 8);
            };
            locate();
            const auto next = [&](FewStage &st) {
                if (load < stop) {
                    const int at = lg * (DIP_INT4_GROUP / 2);
                    const uint8_t *from = from_codes + at, *up = GATED ? from_up + at : nullptr;
                    const size_t step = 8 * half;
                    if (eights == FULL && (lg + 1) * DIP_INT4_GROUP <= p.d_in) {
#pragma unroll
                        for (int i = 0; i < FULL; ++i, from += step) copy16(&st.codes[i][lane], from);
                        if (GATED) {
#pragma unroll
                            for (int i = FULL; i < 8; ++i, up += step) copy16(&st.codes[i][lane], up);
                        }
                        if (lane < 8) copy16(st.scales + 8 * lane, from_scales + (size_t)lg * p.d_out);
                    } else {
                        // (zeros for the inputs that are not there: x is zero there too)
                        const bool mine = lg * DIP_INT4_GROUP + in_quad * 32 < p.d_in;
#pragma unroll 1
                        for (int i = 0; i < eights; ++i, from += step, up += step) {
                            copy16_or_0(&st.codes[i][lane], from, mine);
                            if (GATED) copy16_or_0(&st.codes[FULL + i][lane], up, mine);
                        }
                        if (lane < 8 && lane % FULL < eights) copy16(st.scales + 8 * lane, from_scales + (size_t)lg * p.d_out);
                    }
                    ++load;
                    if (++lg == G && load < stop) {
                        lg = 0;
                        ++lt;
                        locate();
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            int xt = lt, xg = lg;                                           // whose x is loaded next
#pragma unroll
            for (int i = 0; i < STAGES - 1; ++i) next(s.ring[warp][i]);
            uint4 x[NT][4] = {};                                            // (comes straight into registers, a group ahead)
            const __nv_bfloat16 *from_x;
            int tile_rows;
            const auto locate_x = [&] {
                from_x = p.rows + (size_t)(s.tile[xt].row0 + quad) * p.d_in + in_quad * 32;
                tile_rows = s.tile[xt].rows;
            };
            // (the sums of rows that are not there are nobody's, so whatever was here in front may stand for them)
            const auto load_x = [&] {
                const int at = xg * DIP_INT4_GROUP;
                const bool in = at + in_quad * 32 < p.d_in;
#pragma unroll
                for (int m = 0; m < NT; ++m) {
                    const uint4 *from = reinterpret_cast<const uint4 *>(from_x + (size_t)8 * m * p.d_in + at);
                    if (in && 8 * m + quad < tile_rows) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[m][i] = from[i];
                    }
                    if (!in) x[m][0] = x[m][1] = x[m][2] = x[m][3] = make_uint4(0u, 0u, 0u, 0u);
                }
            };
            locate_x();
            load_x();
            float acc[4][NT][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int m = 0; m < NT; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][m][j] = 0.f;
            int slot = 0;
            for (int done = first; done < stop; ++done) {
                asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
                __syncwarp();                           // (also: the unit in front has been read by all lanes)
                const FewStage &st = s.ring[warp][slot];
                next(s.ring[warp][slot == 0 ? STAGES - 1 : slot - 1]);
                const int tile = xt;
                const bool tile_ends = xg + 1 == G || done + 1 == stop;
                uint32_t b[NT][16];
#pragma unroll
                for (int m = 0; m < NT; ++m)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint4 v = x[m][w];
                        b[m][4 * w] = __byte_perm(v.x, v.z, 0x5410);        // inputs 0 and 4 of the word's eight, then 1 and 5, ...
                        b[m][4 * w + 1] = placed(__byte_perm(v.x, v.z, 0x7632));
                        b[m][4 * w + 2] = __byte_perm(v.y, v.w, 0x5410);
                        b[m][4 * w + 3] = placed(__byte_perm(v.y, v.w, 0x7632));
                    }
                if (done + 1 < stop) {
                    if (++xg == G) {
                        xg = 0;
                        ++xt;
                        locate_x();
                    }
                    load_x();
                }
                // (IL sums of 16 outputs side by side: MMAs that wait for one another take 20 cycles each)
                constexpr int IL = 4;
#pragma unroll
                for (int i0 = 0; i0 < 4; i0 += IL) {
                    uint4 q[2 * IL];
#pragma unroll
                    for (int i = 0; i < 2 * IL; ++i) q[i] = st.codes[2 * i0 + i][lane];
                    float d[IL][NT][4];
#pragma unroll
                    for (int w = 0; w < 4; ++w)
#pragma unroll
                        for (int i = 0; i < IL; ++i) {
                            const uint4 lo = q[2 * i], hi = q[2 * i + 1];
                            uint32_t a[4], c[4];
                            int4_pairs(w == 0 ? lo.x : w == 1 ? lo.y : w == 2 ? lo.z : lo.w, a);
                            int4_pairs(w == 0 ? hi.x : w == 1 ? hi.y : w == 2 ? hi.z : hi.w, c);
#pragma unroll
                            for (int m = 0; m < NT; ++m) {
                                if (w == 0) mma_bf16_first(d[i][m], a[0], c[0], a[1], c[1], b[m][0], b[m][1]);
                                else mma_bf16(d[i][m], a[0], c[0], a[1], c[1], b[m][4 * w], b[m][4 * w + 1]);
                                mma_bf16(d[i][m], a[2], c[2], a[3], c[3], b[m][4 * w + 2], b[m][4 * w + 3]);
                            }
                        }
#pragma unroll
                    for (int i = 0; i < IL; ++i) {
                        const __half *sc = st.scales + 16 * (i0 + i) + quad;
                        const float s0 = __half2float(sc[0]) * INT4_PRODUCT, s1 = __half2float(sc[8]) * INT4_PRODUCT;
#pragma unroll
                        for (int m = 0; m < NT; ++m) {
                            acc[i0 + i][m][0] = fmaf(d[i][m][0], s0, acc[i0 + i][m][0]);
                            acc[i0 + i][m][1] = fmaf(d[i][m][1], s0, acc[i0 + i][m][1]);
                            acc[i0 + i][m][2] = fmaf(d[i][m][2], s1, acc[i0 + i][m][2]);
                            acc[i0 + i][m][3] = fmaf(d[i][m][3], s1, acc[i0 + i][m][3]);
                        }
                    }
                }
                slot = slot == STAGES - 1 ? 0 : slot + 1;
                if (tile_ends) {
                    // this warp's part of the tile
                    float(*to)[IF_PITCH] = s.part[warp + tile];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int m = 0; m < NT; ++m)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                to[8 * m + 2 * in_quad + (j & 1)][16 * i + quad + 8 * (j >> 1)] = acc[i][m][j];
                                acc[i][m][j] = 0.f;
                            }
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
        __syncthreads();
        // Sums of 4 neighbouring outputs of a row per thread; gate/up: of gate or up, the neighbouring thread has the other one.
        constexpr int QUADS = IF_OUTS / 4, PER_TILE = 8 * NT * QUADS;
        constexpr size_t PART = (size_t)8 * NT * IF_OUTS;
        const auto leave = [&](const FewTile &t, int r, int c, const float4 &v) {
            const size_t row = (size_t)(t.row0 + r) * p.d_out;
            const int o = t.out0 + c;
            if (GATED) {
                // (h is rounded once, to bfloat16: it is an operand of the next product, whose MMAs take no more)
                float4 u;
                u.x = __shfl_down_sync(0xffffffffu, v.x, 1);
                u.y = __shfl_down_sync(0xffffffffu, v.y, 1);
                u.z = __shfl_down_sync(0xffffffffu, v.z, 1);
                u.w = __shfl_down_sync(0xffffffffu, v.w, 1);
                if (r < t.rows && tid % 2 == 0 && o < p.d_out)
                    *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.out) + row + o) =
                        bf16x4(silu_f32(v.x) * u.x, silu_f32(v.y) * u.y, silu_f32(v.z) * u.z, silu_f32(v.w) * u.w);
            } else if (r < t.rows && o < p.d_out) {
                if (p.out_f32) *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + row + o) = v;
                else *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.out) + row + o) = bf16x4(v.x, v.y, v.z, v.w);
            }
        };
        // (whole warps: PER_TILE and the number of threads are multiples of 32)
        for (int i = tid; i < (t1 - t0) * PER_TILE; i += IF_THREADS<NT>) {
            const int k = i / PER_TILE, q = i % QUADS, r = i / QUADS % (8 * NT), c = GATED ? q / 2 * 4 + q % 2 * (IF_OUTS / 2) : q * 4;
            const FewTile t = s.tile[k];
            float4 v = {};
            if (r < t.rows) {
                for (int w = t.w0; w <= t.w1; ++w) {
                    const float4 a = *reinterpret_cast<const float4 *>(&s.part[w + k][r][c]);
                    v.x += a.x;
                    v.y += a.y;
                    v.z += a.z;
                    v.w += a.w;
                }
            }
            // A tile that is cut: a block's first one may have begun in front of it, its last one may go on behind it.
            if (t.b0 == t.b1) leave(t, r, c, v);
            else if (r < t.rows) reinterpret_cast<float4 *>(p.partials + (2 * (size_t)blockIdx.x + ((int)blockIdx.x == t.b0)) * PART)[r * QUADS + q] = v;
        }
        for (int k = 0; k < t1 - t0; k = k == t1 - t0 - 1 ? k + 1 : t1 - t0 - 1) {           // (the first one and the last one)
            const FewTile t = s.tile[k];
            if (t.b0 == t.b1) continue;
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                s.last = atomicAdd(p.tickets + t.b0, 1u) == (unsigned)(t.b1 - t.b0);
                if (s.last) p.tickets[t.b0] = 0u;
                __threadfence();
            }
            __syncthreads();
            if (!s.last) continue;
            for (int i = tid; i < PER_TILE; i += IF_THREADS<NT>) {
                const int q = i % QUADS, r = i / QUADS, c = GATED ? q / 2 * 4 + q % 2 * (IF_OUTS / 2) : q * 4;
                float4 v = {};
                if (r < t.rows) {
                    for (int b = t.b0; b <= t.b1; ++b) {
                        const float4 a = __ldcg(reinterpret_cast<const float4 *>(p.partials + (2 * (size_t)b + (b == t.b0)) * PART) + r * QUADS + q);
                        v.x += a.x;
                        v.y += a.y;
                        v.z += a.z;
                        v.w += a.w;
                    }
                }
                leave(t, r, c, v);
            }
        }
        u0 = end;
        __syncthreads();                        // (the parts have been read)
    }
    DIP_TRACE_MAX(p.tr, 2);
}

template <bool GATED, int NT>
cudaError_t launch(dip_ctx *ctx, int ctas, cudaStream_t stream, const FewParams &p)
{
    static dip_per_device_once once;
    constexpr size_t smem = sizeof(FewSmem<NT>);
    static_assert(smem <= 227 * 1024, "fits a CTA's shared memory");
    const cudaError_t e = dip_raise_smem_limit(once, ctx->device, int4_few_kernel<GATED, NT>, smem);
    if (e != cudaSuccess) return e;
    return dip_launch_pdl(int4_few_kernel<GATED, NT>, dim3(ctas), dim3(IF_THREADS<NT>), smem, stream, p);
}

}  // namespace

dip_status dip_launch_int4_few(dip_ctx *ctx, const dip_grouped_matrix &w, const dip_grouped_matrix *up, const void *rows, int n_rows,
                               const int32_t *offset, void *out, bool out_f32, cudaStream_t stream)
{
    const int met = min(w.n_experts, n_rows);
    FewParams p = {};
    p.codes = static_cast<const uint8_t *>(w.values);
    p.scales = static_cast<const __half *>(w.scales);
    if (up) {
        p.up_codes = static_cast<const uint8_t *>(up->values);
        p.up_scales = static_cast<const __half *>(up->scales);
    }
    p.rows = static_cast<const __nv_bfloat16 *>(rows);
    p.offset = offset;
    p.n_experts = w.n_experts;
    p.d_out = w.d_out;
    p.d_in = w.d_in;
    p.n_rows = n_rows;
    p.groups = (w.d_in + DIP_INT4_GROUP - 1) / DIP_INT4_GROUP;
    const int width = up ? IF_OUTS / 2 : IF_OUTS;
    p.n_cols = (w.d_out + width - 1) / width;
    p.out = out;
    p.out_f32 = out_f32;
    p.partials = ctx->partials;
    p.tickets = ctx->group_tickets;
    p.tr = dip_trace_slot(ctx, up ? 10 : 11);
    const bool wide = n_rows > 8 * met;         // (9 rows and more at a time take as long as 16)
    const long long most = ((long long)(n_rows + 7) / 8 + met) * p.n_cols * p.groups;
    const int ctas = (int)min((long long)ctx->sm_count, most);
    DIP_CUDA_TRY(ctx, up ? (wide ? launch<true, 2>(ctx, ctas, stream, p) : launch<true, 1>(ctx, ctas, stream, p))
                         : (wide ? launch<false, 2>(ctx, ctas, stream, p) : launch<false, 1>(ctx, ctas, stream, p)));
    return DIP_OK;
}
