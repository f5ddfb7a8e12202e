// Products of groups of few rows with 4-bit weights: y[r] = W[e(r)] rows[r], h[r] = silu(Wg[e(r)] rows[r]) * (Wu[e(r)] rows[r]), where
// W[o][i] = (code - 8) * S[i / 128][o].  Per group of 128 input indices the products code * x are exact in binary32 and are summed by the
// tensor cores (m16n8k16: 16 outputs x 16 inputs x 8 rows of bfloat16); each group's sum is then multiplied by its scale into the output's
// binary32 sum.  Nothing but y is rounded to fewer bits.
//
// Bound by the stream of codes, so what matters is that every SM has enough of it under way and that the ALUs, which turn codes into
// bfloat16, keep up:
//   * A unit is 64 outputs (gate/up: 32 of each) by one group: 4 KB of codes, 64 bytes of a row at a time.  Each warp has a ring of
//     units that it fills with asynchronous copies of its own and waits for by itself; a lane reads back what it copied.
//   * A lane's 16 bytes of a row are 32 consecutive codes, and the sums of a group do not depend on the order of its inputs, so the four lanes
//     of a quad simply take a quarter of the group each, and MMA j takes the codes that one AND brings out of a word: nibbles s and s + 4,
//     left at the bottom of two bfloat16 of 128 (128 + code is exact there, 136 is subtracted).  x is paired alike.
//   * All units, tile after tile, are dealt out to the blocks in equal runs, and a block's to its warps: whatever the sizes, nobody has
//     more than a unit too many.  Where whole tiles are hardly worse for the blocks, they stay whole: parts of a tile that meet in
//     the workspace cost a write, a count and a read (the block that comes last adds them up in order; nobody waits).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "float8.cuh"
#include "gemv_common.cuh"
#include "int4_codes.cuh"

namespace {

constexpr int IF_WARPS = 8, IF_THREADS = IF_WARPS * 32;
constexpr int IF_OUTS = 64;                 // outputs of a tile (gate/up: as many sums, of half as many outputs)
constexpr int IF_PITCH = IF_OUTS + 4;       // floats of a row of partial sums in shared memory (conflict-free)
constexpr int IF_TILES = 4;                 // tiles that a block has in hand at a time
constexpr int IF_JOIN = 24;                 // units' worth of time that parts of a tile take to meet

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

template <int NT> struct __align__(16) FewStage {
    uint4 codes[8][32];                     // tile of 16 outputs, half of it; lane
    uint4 x[NT][4][32];
    __half scales[IF_OUTS];
    static constexpr int COUNT = NT == 1 ? 4 : 2;   // of a warp (what shared memory has room for)
};

template <int NT> struct __align__(16) FewSmem {
    FewStage<NT> ring[IF_WARPS][FewStage<NT>::COUNT];
    float part[IF_WARPS + IF_TILES][8 * NT][IF_PITCH];
    int start[DIP_MAX_EXPERTS + 1];         // first row of each expert
    int tiles[DIP_MAX_EXPERTS + 1];         // tiles in front of it
    int last;
};

// 16 bytes to shared memory, asynchronously; zeros instead where there is nothing to read.
__device__ __forceinline__ void copy16(void *dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A tile: 8 * NT rows of one expert, 64 sums of each.
struct FewTile {
    int expert, row0, rows, out0;
};

template <bool GATED, int NT>
__device__ __forceinline__ FewTile few_tile(const FewParams &p, const FewSmem<NT> &s, int tile)
{
    int lo = 0, hi = p.n_experts;           // the expert with tiles[e] <= tile < tiles[e + 1]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.tiles[mid] <= tile) lo = mid;
        else hi = mid;
    }
    const int n = s.start[lo + 1] - s.start[lo], chunks = (n + 8 * NT - 1) / (8 * NT), in = tile - s.tiles[lo], col = in / chunks;
    const int first = (in - col * chunks) * 8 * NT;
    return {lo, s.start[lo] + first, min(8 * NT, n - first), col * (GATED ? IF_OUTS / 2 : IF_OUTS)};
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

// Of n units dealt out to `parts` in equal runs: where run i starts, and whose a unit is (no run is empty: parts <= n).
__device__ __forceinline__ long long run_start(long long n, int parts, int i) { return n * i / parts; }
__device__ __forceinline__ int run_of(long long n, int parts, long long unit) { return (int)(((unit + 1) * parts - 1) / n); }

template <bool GATED, int NT>
__global__ void __launch_bounds__(IF_THREADS, 1)
int4_few_kernel(const FewParams p)
{
    extern __shared__ unsigned char if_smem_raw[];
    FewSmem<NT> &s = *reinterpret_cast<FewSmem<NT> *>(if_smem_raw);
    constexpr int STAGES = FewStage<NT>::COUNT;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, quad = lane >> 2, in_quad = lane & 3;
    DIP_TRACE_MIN(p.tr, 0);
    dip_grid_dependency_wait();
    DIP_TRACE_MIN(p.tr, 1);
    if (warp == 0) few_plan(p, s);
    __syncthreads();
    dip_launch_dependents();

    const int tiles = s.tiles[p.n_experts], G = p.groups, blocks = gridDim.x;
    const long long units = (long long)tiles * G;
    const int whole_each = (tiles + blocks - 1) / blocks;
    const bool whole = (long long)whole_each * G <= units / blocks + IF_JOIN;
    const int parts = (int)min((long long)blocks, units);
    long long u0 = 0, u1 = 0;               // this block's units
    if (whole) {
        u0 = min(units, (long long)run_start(tiles, blocks, blockIdx.x) * G);
        u1 = min(units, (long long)run_start(tiles, blocks, blockIdx.x + 1) * G);
    } else if ((int)blockIdx.x < parts) {
        u0 = run_start(units, parts, blockIdx.x);
        u1 = run_start(units, parts, blockIdx.x + 1);
    }

    while (u0 < u1) {
        // the next tiles
        const int t0 = (int)(u0 / G), t1 = min(t0 + IF_TILES, (int)((u1 + G - 1) / G));
        const long long end = min(u1, (long long)t1 * G);
        const int n = (int)(end - u0), warps = min(IF_WARPS, n);
        if (warp < warps) {
            int load = (int)run_start(n, warps, warp), done = load;
            const int stop = (int)run_start(n, warps, warp + 1);
            // where the copies are
            int lt = (int)((u0 + load) / G), lg = (int)((u0 + load) - (long long)lt * G);
            FewTile t = few_tile<GATED, NT>(p, s, lt);
            const auto copy = [&](FewStage<NT> &st) {
                const int left = p.d_in - lg * DIP_INT4_GROUP;               // inputs from this group on
                const bool mine = in_quad * 32 < left;
                const size_t half = (size_t)p.d_in / 2, at = (size_t)lg * (DIP_INT4_GROUP / 2) + in_quad * 16;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool up = GATED && i >= 4;
                    const int o = t.out0 + (GATED ? i & 3 : i) * 8 + quad;
                    const uint8_t *from = up ? p.up_codes : p.codes;
                    copy16(&st.codes[i][lane], mine ? from + ((size_t)t.expert * p.d_out + min(o, p.d_out - 1)) * half + at : from, mine);
                }
#pragma unroll
                for (int m = 0; m < NT; ++m) {
                    const bool there = mine && 8 * m + quad < t.rows;
                    const __nv_bfloat16 *from = p.rows + (there ? (size_t)(t.row0 + 8 * m + quad) * p.d_in + lg * DIP_INT4_GROUP + in_quad * 32 : 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) copy16(&st.x[m][i][lane], there ? from + 8 * i : from, there);
                }
                if (lane < 8) {
                    const bool up = GATED && lane >= 4;
                    const int o = t.out0 + (GATED ? lane & 3 : lane) * 8;
                    const __half *from = up ? p.up_scales : p.scales;
                    copy16(st.scales + 8 * lane, o < p.d_out ? from + ((size_t)t.expert * G + lg) * p.d_out + o : from, o < p.d_out);
                }
            };
            const auto next = [&](int slot) {
                if (load < stop) {
                    copy(s.ring[warp][slot]);
                    ++load;
                    if (++lg == G && load < stop) {
                        lg = 0;
                        t = few_tile<GATED, NT>(p, s, ++lt);
                    }
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
#pragma unroll
            for (int i = 0; i < STAGES - 1; ++i) next(i);
            float acc[4][NT][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int m = 0; m < NT; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][m][j] = 0.f;
            int tile = (int)((u0 + done) / G), g = (int)((u0 + done) - (long long)tile * G), slot = 0;
            while (done < stop) {
                asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
                __syncwarp();                           // (also: the unit in front has been read by all lanes)
                next((slot + STAGES - 1) % STAGES);
                const FewStage<NT> &st = s.ring[warp][slot];
                uint32_t b[NT][16];
#pragma unroll
                for (int m = 0; m < NT; ++m)
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint4 v = st.x[m][w][lane];
                        b[m][4 * w] = __byte_perm(v.x, v.z, 0x5410);        // inputs 0 and 4 of the word's eight, then 1 and 5, ...
                        b[m][4 * w + 1] = __byte_perm(v.x, v.z, 0x7632);
                        b[m][4 * w + 2] = __byte_perm(v.y, v.w, 0x5410);
                        b[m][4 * w + 3] = __byte_perm(v.y, v.w, 0x7632);
                    }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 lo = st.codes[2 * i][lane], hi = st.codes[2 * i + 1][lane];
                    float d[NT][4];
#pragma unroll
                    for (int m = 0; m < NT; ++m) d[m][0] = d[m][1] = d[m][2] = d[m][3] = 0.f;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        uint32_t a[4], c[4];
                        int4_pairs(w == 0 ? lo.x : w == 1 ? lo.y : w == 2 ? lo.z : lo.w, a);
                        int4_pairs(w == 0 ? hi.x : w == 1 ? hi.y : w == 2 ? hi.z : hi.w, c);
#pragma unroll
                        for (int m = 0; m < NT; ++m) {
                            mma_bf16(d[m], a[0], c[0], a[1], c[1], b[m][4 * w], b[m][4 * w + 1]);
                            mma_bf16(d[m], a[2], c[2], a[3], c[3], b[m][4 * w + 2], b[m][4 * w + 3]);
                        }
                    }
                    const float s0 = __half2float(st.scales[16 * i + quad]), s1 = __half2float(st.scales[16 * i + 8 + quad]);
#pragma unroll
                    for (int m = 0; m < NT; ++m) {
                        acc[i][m][0] = fmaf(d[m][0], s0, acc[i][m][0]);
                        acc[i][m][1] = fmaf(d[m][1], s0, acc[i][m][1]);
                        acc[i][m][2] = fmaf(d[m][2], s1, acc[i][m][2]);
                        acc[i][m][3] = fmaf(d[m][3], s1, acc[i][m][3]);
                    }
                }
                slot = (slot + 1) % STAGES;
                ++done;
                if (++g == G || done == stop) {
                    // this warp's part of the tile
                    float(*to)[IF_PITCH] = s.part[warp + tile - t0];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int m = 0; m < NT; ++m)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                to[8 * m + 2 * in_quad + (j & 1)][16 * i + quad + 8 * (j >> 1)] = acc[i][m][j];
                                acc[i][m][j] = 0.f;
                            }
                    g = 0;
                    ++tile;
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
        __syncthreads();
        for (int tile = t0; tile < t1; ++tile) {
            const FewTile t = few_tile<GATED, NT>(p, s, tile);
            const long long a = max((long long)tile * G, u0) - u0, z = min((long long)(tile + 1) * G, end) - u0;
            const int w0 = run_of(n, warps, a), w1 = run_of(n, warps, z - 1);
            const bool cut = z - a < G;
            // sums of 4 neighbouring outputs of one row; gate/up: 4 of each
            constexpr int QUADS = IF_OUTS / 4;
            const int r = tid / QUADS, c = (GATED ? tid % QUADS / 2 * 4 + tid % 2 * (IF_OUTS / 2) : tid % QUADS * 4);
            const int b0 = cut ? run_of(units, parts, (long long)tile * G) : 0, b1 = cut ? run_of(units, parts, (long long)(tile + 1) * G - 1) : 0;
            float4 v = {};
            if (r < t.rows) {
                for (int w = w0; w <= w1; ++w) {
                    const float4 q = *reinterpret_cast<const float4 *>(&s.part[w + tile - t0][r][c]);
                    v.x += q.x;
                    v.y += q.y;
                    v.z += q.z;
                    v.w += q.w;
                }
            }
            if (cut) {
                constexpr size_t PART = (size_t)8 * NT * IF_OUTS;
                // a block's first tile may have begun in front of it, its last one may go on behind it
                const auto part_at = [&](int b) {
                    return reinterpret_cast<float4 *>(p.partials + (2 * (size_t)b + (b == b0 ? 1 : 0)) * PART) + r * QUADS + c / 4;
                };
                if (r < t.rows) *part_at(blockIdx.x) = v;
                __threadfence();
                __syncthreads();
                if (tid == 0) {
                    s.last = atomicAdd(p.tickets + b0, 1u) == (unsigned)(b1 - b0);
                    if (s.last) p.tickets[b0] = 0u;
                    __threadfence();
                }
                __syncthreads();
                if (!s.last) continue;
                v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (r < t.rows) {
                    for (int b = b0; b <= b1; ++b) {
                        const float4 q = __ldcg(part_at(b));
                        v.x += q.x;
                        v.y += q.y;
                        v.z += q.z;
                        v.w += q.w;
                    }
                }
            }
            const size_t row = (size_t)(t.row0 + r) * p.d_out;
            if (GATED) {
                // (the neighbouring thread has the other one of gate and up)
                float4 u;
                u.x = __shfl_down_sync(0xffffffffu, v.x, 1);
                u.y = __shfl_down_sync(0xffffffffu, v.y, 1);
                u.z = __shfl_down_sync(0xffffffffu, v.z, 1);
                u.w = __shfl_down_sync(0xffffffffu, v.w, 1);
                if (r < t.rows && tid % 2 == 0 && t.out0 + c < p.d_out)
                    *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.out) + row + t.out0 + c) =
                        bf16x4(silu_f32(v.x) * u.x, silu_f32(v.y) * u.y, silu_f32(v.z) * u.z, silu_f32(v.w) * u.w);
            } else if (r < t.rows && t.out0 + c < p.d_out) {
                if (p.out_f32) *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + row + t.out0 + c) = v;
                else *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(p.out) + row + t.out0 + c) = bf16x4(v.x, v.y, v.z, v.w);
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
    static_assert(8 * NT * (IF_OUTS / 4) <= IF_THREADS, "a thread for each four sums");
    const cudaError_t e = dip_raise_smem_limit(once, ctx->device, int4_few_kernel<GATED, NT>, smem);
    if (e != cudaSuccess) return e;
    return dip_launch_pdl(int4_few_kernel<GATED, NT>, dim3(ctas), dim3(IF_THREADS), smem, stream, p);
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
    const bool wide = n_rows > 8 * met;
    const long long most = ((long long)(n_rows + 7) / 8 + met) * p.n_cols * p.groups;
    const int ctas = (int)min((long long)ctx->sm_count, most);
    DIP_CUDA_TRY(ctx, up ? (wide ? launch<true, 2>(ctx, ctas, stream, p) : launch<true, 1>(ctx, ctas, stream, p))
                         : (wide ? launch<false, 2>(ctx, ctas, stream, p) : launch<false, 1>(ctx, ctas, stream, p)));
    return DIP_OK;
}
