// The router of a mixture, and the rows on their way into the grouped products and out of them.
//
// Choice: a warp per token holds the token's logits in registers (E / 32 per lane) and takes the largest top_k times: one
// warp-wide maximum over order-preserving integers, one warp-wide minimum over the indices that hold it (ties: lowest).  A bfloat16
// logit's integer has 16 bits and shares a word with its index, which makes one maximum of both.  Up to four logits a lane are sorted
// first, so that a choice takes a lane's first one and shifts the others up.
// Grouping: row = first row of the expert + tokens in front that chose it.  A block has up to DIP_ROUTE_TOKENS tokens and a bit set
// of them per expert, so a rank within the block is a popcount; nothing depends on the order of atomics.  A token per warp of one
// block is one launch.  More are two: the blocks leave their counts, and every block of the second launch
// adds up the counts in front of its own (blocks^2 * E words out of L2; 16384 tokens, 128 experts: 8 MB).  Blocks have a token per
// warp, and four from 128 blocks on, which keeps that in bounds (128 tokens in one block took 10.5 us, in four 5.3).  From
// 128 blocks of four on a launch in between does the adding (65536 tokens, 256 experts: 108 us without).
// Bound by latency for a token, by the trips to memory between the launches for a prompt.
#include <cuda_bf16.h>

#include "common.cuh"
#include "float8.cuh"
#include "gemv_common.cuh"

namespace {

constexpr int RT_THREADS = 1024, RT_WARPS = RT_THREADS / 32;
constexpr int RT_WORDS = DIP_ROUTE_TOKENS / 32;
constexpr uint32_t RT_ALL = 0xffffffffu;

struct RouteParams {
    const void *logits;
    int n_tokens, n_experts, top_k, renormalize, block_tokens, added;
    int32_t *expert;
    float *weight;
    int32_t *offset, *row_token, *token_row;
    int32_t *counts;         // [blocks][DIP_MAX_EXPERTS]
};

struct RouteSmem {
    uint32_t chosen[DIP_MAX_EXPERTS][RT_WORDS];   // tokens of this block that chose the expert
    int32_t start[DIP_MAX_EXPERTS];               // first row of this block's tokens in the expert's group
    int32_t total[DIP_MAX_EXPERTS];
    int32_t warp_sum[RT_WARPS];
};

// Order-preserving image of a logit; 0: closed.  (-0 and 0 are equal.)
__device__ __forceinline__ uint32_t route_key(float v)
{
    v += 0.f;
    if (!(v > -INFINITY)) return 0u;
    const uint32_t b = __float_as_uint(v);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float route_value(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key); }
__device__ __forceinline__ float route_part(uint32_t key, float high)
{
    if (key == 0u) return 0.f;
    const float v = route_value(key);
    return high == INFINITY ? (v == INFINITY ? 1.f : 0.f) : expf(v - high);
}

// The image of a logit out of a word that it shares with its index.
template <bool BF16>
__device__ __forceinline__ uint32_t unpacked(uint32_t key)
{
    return !BF16 || key == 0u ? key : (key & 0x80000000u) ? key & 0xffff0000u : key | 0xffffu;
}

// The greater of two keys first; among equals the lower index (bfloat16 keys have it in them).
template <bool BF16>
__device__ __forceinline__ void first_greater(uint32_t &a, uint32_t &b, int &ia, int &ib)
{
    const uint32_t hi = max(a, b), lo = min(a, b);
    if (!BF16) {
        const bool swap = b > a || (b == a && ib < ia);
        const int i = ia;
        ia = swap ? ib : ia;
        ib = swap ? i : ib;
    }
    a = hi;
    b = lo;
}

// Tokens t0 + 32 m (m < M, below n) of a block, one warp: experts and weights, and the tokens' bits in the sets of their experts.  M of
// them side by side, because one alone waits: for its logits, and for each choice's two trips through all lanes.
template <int NV, int M, bool BF16>
__device__ __forceinline__ void route_tokens(const RouteParams &p, int first, int bit0, int n, RouteSmem &s)
{
    const int lane = threadIdx.x & 31;
    uint32_t key[M][NV], most[M];
    float raw[M][NV];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int e = lane + 32 * i;
            raw[m][i] = -INFINITY;
            if (e < p.n_experts && bit0 + 32 * m < n) {
                const size_t at = (size_t)(first + bit0 + 32 * m) * p.n_experts + e;
                raw[m][i] = BF16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p.logits)[at]) : static_cast<const float *>(p.logits)[at];
            }
        }
    float high[M], sum[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
        most[m] = 0u;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            key[m][i] = route_key(raw[m][i]);
            if (BF16 && key[m][i]) key[m][i] = (key[m][i] & 0xffff0000u) | (0xffffu - (lane + 32 * i));
            most[m] = max(most[m], key[m][i]);
        }
    }
#pragma unroll
    for (int m = 0; m < M; ++m) most[m] = __reduce_max_sync(RT_ALL, most[m]);
#pragma unroll
    for (int m = 0; m < M; ++m) {
        high[m] = route_value(unpacked<BF16>(most[m]));
        sum[m] = 0.f;
        if (!p.renormalize) {
#pragma unroll
            for (int i = 0; i < NV; ++i) sum[m] += route_part(unpacked<BF16>(key[m][i]), high[m]);
        }
    }
    uint32_t mine[M];                             // choice `lane`
    int mine_e[M];
    int index[M][NV];                             // (BF16: in the keys)
#pragma unroll
    for (int m = 0; m < M; ++m) {
        mine[m] = 0u;
        mine_e[m] = -1;
#pragma unroll
        for (int i = 0; i < NV; ++i) index[m][i] = lane + 32 * i;
        if (NV == 2) first_greater<BF16>(key[m][0], key[m][NV - 1], index[m][0], index[m][NV - 1]);
        if (NV == 4) {
            constexpr int a[5] = {0, 2, 0, 1, 1}, b[5] = {1, 3, 2, 3, 2};
#pragma unroll
            for (int q = 0; q < 5; ++q) first_greater<BF16>(key[m][a[q] % NV], key[m][b[q] % NV], index[m][a[q] % NV], index[m][b[q] % NV]);
        }
    }
    constexpr bool SORTED = NV <= 4;
    for (int j = 0; j < p.top_k; ++j) {
        unsigned at[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
            at[m] = 0xffffu - (most[m] & 0xffffu);
            if (!BF16) {
                at[m] = 0x7fffffffu;
#pragma unroll
                for (int i = SORTED ? 0 : NV - 1; i >= 0; --i)
                    if (key[m][i] == most[m]) at[m] = index[m][i];
            }
        }
        if (!BF16) {
#pragma unroll
            for (int m = 0; m < M; ++m) at[m] = __reduce_min_sync(RT_ALL, at[m]);
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int e = most[m] ? (int)at[m] : -1;          // (no expert is left: closed ones have the key 0)
            if (lane == j) {
                mine[m] = most[m];
                mine_e[m] = e;
            }
            if (SORTED) {
                if ((e & 31) == lane) {                       // (with none left: zeros move up)
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        key[m][i] = i + 1 < NV ? key[m][(i + 1) % NV] : 0u;
                        index[m][i] = index[m][(i + 1) % NV];
                    }
                }
                most[m] = key[m][0];
            } else {
                most[m] = 0u;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (index[m][i] == e) key[m][i] = 0u;
                    most[m] = max(most[m], key[m][i]);
                }
            }
        }
#pragma unroll
        for (int m = 0; m < M; ++m) most[m] = __reduce_max_sync(RT_ALL, most[m]);
    }
    float part[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
        part[m] = route_part(unpacked<BF16>(mine[m]), high[m]);
        if (p.renormalize) sum[m] = part[m];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int m = 0; m < M; ++m) sum[m] += __shfl_xor_sync(RT_ALL, sum[m], o);
#pragma unroll
    for (int m = 0; m < M; ++m) {
        const int bit = bit0 + 32 * m;
        if (lane < p.top_k && bit < n) {
            const size_t to = (size_t)(first + bit) * p.top_k + lane;
            p.expert[to] = mine_e[m];
            p.weight[to] = mine_e[m] >= 0 ? part[m] / sum[m] : 0.f;
            if (mine_e[m] >= 0) atomicOr(&s.chosen[mine_e[m]][bit >> 5], 1u << (bit & 31));
        }
    }
}

// start[e] += exclusive prefix of total[0 .. E); block 0 also writes the offsets.  All threads.
__device__ __forceinline__ void route_offsets(const RouteParams &p, RouteSmem &s)
{
    static_assert(RT_THREADS >= DIP_MAX_EXPERTS, "a thread per expert");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n = tid < p.n_experts ? s.total[tid] : 0;
    int incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(RT_ALL, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) s.warp_sum[warp] = incl;
    __syncthreads();
    const int first = (int)__reduce_add_sync(RT_ALL, lane < warp ? (unsigned)s.warp_sum[lane] : 0u) + incl - n;
    if (tid < p.n_experts) {
        s.start[tid] += first;
        if (blockIdx.x == 0) {
            p.offset[tid] = first;
            if (tid == p.n_experts - 1) p.offset[tid + 1] = first + n;
        }
    }
    __syncthreads();
}

// Rows of this block's choices.
__device__ __forceinline__ void route_rows(const RouteParams &p, const RouteSmem &s, int t0, int n)
{
    for (int i = threadIdx.x; i < n * p.top_k; i += RT_THREADS) {
        const int bit = i / p.top_k;
        const size_t at = (size_t)t0 * p.top_k + i;
        const int e = p.expert[at];
        int row = -1;
        if (e >= 0) {
            row = s.start[e];
#pragma unroll
            for (int w = 0; w < RT_WORDS; ++w) {
                const int below = bit - 32 * w;
                row += __popc(s.chosen[e][w] & (below >= 32 ? RT_ALL : below > 0 ? (1u << below) - 1u : 0u));
            }
            p.row_token[row] = t0 + bit;
        }
        p.token_row[at] = row;
    }
}

__device__ __forceinline__ void route_clear(const RouteParams &p, RouteSmem &s)
{
    for (int i = threadIdx.x; i < p.n_experts * RT_WORDS; i += RT_THREADS) (&s.chosen[0][0])[i] = 0u;
    for (int i = threadIdx.x; i < p.n_experts; i += RT_THREADS) s.start[i] = s.total[i] = 0;
    __syncthreads();
}

template <int NV, bool BF16>
__global__ void __launch_bounds__(RT_THREADS, 1) route_choose_kernel(const RouteParams p)
{
    __shared__ RouteSmem s;
    const int t0 = blockIdx.x * p.block_tokens, n = min(p.block_tokens, p.n_tokens - t0);
    route_clear(p, s);
    dip_grid_dependency_wait();
    dip_launch_dependents();
    const int warp = threadIdx.x >> 5;
    static_assert(DIP_ROUTE_TOKENS == 4 * RT_WARPS, "four tokens a warp");
    if (n <= RT_WARPS) {
        if (warp < n) route_tokens<NV, 1, BF16>(p, t0, warp, n, s);
    } else if (NV <= 8) {
        route_tokens<NV, 4, BF16>(p, t0, warp, n, s);
    } else {                                      // (64 registers each at 1024 threads: eight logits a lane, four tokens, spill 24 to 32 bytes of them)
        for (int bit = warp; bit < n; bit += RT_WARPS) route_tokens<NV, 1, BF16>(p, t0, bit, n, s);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.n_experts; e += RT_THREADS) {
        int c = 0;
#pragma unroll
        for (int w = 0; w < RT_WORDS; ++w) c += __popc(s.chosen[e][w]);
        s.total[e] = c;
        if (gridDim.x > 1) p.counts[(size_t)blockIdx.x * DIP_MAX_EXPERTS + e] = c;
    }
    if (gridDim.x > 1) return;
    __syncthreads();
    route_offsets(p, s);
    route_rows(p, s, t0, n);
}

// counts[b][e] becomes the sum of those in front of it, and the row behind the last the sum of all.  A block per 32 experts, a lane each;
// a warp has every 32nd part of the rows.
__global__ void __launch_bounds__(RT_THREADS, 1) route_add_kernel(const RouteParams p, int blocks)
{
    __shared__ int32_t part[RT_WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane, each = (blocks + RT_WARPS - 1) / RT_WARPS;
    const int b0 = min(warp * each, blocks), b1 = min(b0 + each, blocks);
    int32_t *c = p.counts + min(e, DIP_MAX_EXPERTS - 1);
    dip_grid_dependency_wait();
    dip_launch_dependents();
    int sum = 0;
#pragma unroll 4
    for (int b = b0; b < b1; ++b) sum += c[(size_t)b * DIP_MAX_EXPERTS];
    part[warp][lane] = sum;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < RT_WARPS; ++w) {
        if (w == warp) before = all;
        all += part[w][lane];
    }
    if (e >= p.n_experts) return;
    for (int b = b0; b < b1; ++b) {
        const int n = c[(size_t)b * DIP_MAX_EXPERTS];
        c[(size_t)b * DIP_MAX_EXPERTS] = before;
        before += n;
    }
    if (warp == 0) c[(size_t)blocks * DIP_MAX_EXPERTS] = all;
}

__global__ void __launch_bounds__(RT_THREADS, 1) route_rows_kernel(const RouteParams p)
{
    __shared__ RouteSmem s;
    const int t0 = blockIdx.x * p.block_tokens, n = min(p.block_tokens, p.n_tokens - t0);
    route_clear(p, s);
    dip_grid_dependency_wait();
    dip_launch_dependents();
    for (int i = threadIdx.x; i < n * p.top_k; i += RT_THREADS) {
        const int e = p.expert[(size_t)t0 * p.top_k + i], bit = i / p.top_k;
        if (e >= 0) atomicOr(&s.chosen[e][bit >> 5], 1u << (bit & 31));
    }
    // all blocks' counts, and those in front of this block
    const int width = p.n_experts <= 32 ? 32 : p.n_experts <= 64 ? 64 : p.n_experts <= 128 ? 128 : p.n_experts <= 256 ? 256 : 512;
    const int e = threadIdx.x % width;
    if (p.added) {
        if (threadIdx.x < p.n_experts) {
            s.start[threadIdx.x] = p.counts[(size_t)blockIdx.x * DIP_MAX_EXPERTS + threadIdx.x];
            s.total[threadIdx.x] = p.counts[(size_t)gridDim.x * DIP_MAX_EXPERTS + threadIdx.x];
        }
    } else if (e < p.n_experts) {
        int total = 0, before = 0;
#pragma unroll 8
        for (int b = threadIdx.x / width; b < (int)gridDim.x; b += RT_THREADS / width) {
            const int c = p.counts[(size_t)b * DIP_MAX_EXPERTS + e];
            total += c;
            if (b < (int)blockIdx.x) before += c;
        }
        atomicAdd(&s.total[e], total);
        atomicAdd(&s.start[e], before);
    }
    __syncthreads();
    route_offsets(p, s);
    route_rows(p, s, t0, n);
}

// ---- rows into their places ----
struct StageParams {
    const uint4 *x;            // [n_tokens][d / 8]
    int n_tokens, n_rows, d;
    const int32_t *row_token;  // nullptr: row r is token r
    const int32_t *end;        // offset + n_experts
    void *rows;
    float *scales;
};

// A piece of a row is 256 columns, eight to a lane: 16 lanes are a block of 128.  A warp takes four pieces of a row, whose loads go
// out together.  Copies are bound by memory: 8192 tokens of 5120 columns take 27.8 us (6.0 TB/s).  To e4m3 it is the quotients: 37.7 us for 127 MB;
// with products by 1 / scale, which come out a code off now and then, 25.4.
constexpr int ST_PIECES = 4;
template <bool FP8>
__global__ void __launch_bounds__(256) stage_rows_kernel(const StageParams p)
{
    dip_grid_dependency_wait();
    dip_launch_dependents();
    const int lane = threadIdx.x & 31, groups = (p.d + 256 * ST_PIECES - 1) / (256 * ST_PIECES), blocks = (p.d + DIP_FP8_BLOCK - 1) / DIP_FP8_BLOCK;
    const int n = (p.end ? max(0, min(*p.end, p.n_rows)) : p.n_rows) * groups;     // (2^20 rows of up to 32 groups)
    for (int i = blockIdx.x * 8 + (threadIdx.x >> 5); i < n; i += gridDim.x * 8) {
        const int r = i / groups, c0 = (i - r * groups) * (256 * ST_PIECES) + lane * 8;
        const int t = p.row_token ? p.row_token[r] : r;
        uint4 v[ST_PIECES];
#pragma unroll
        for (int q = 0; q < ST_PIECES; ++q) {
            const int c = c0 + 256 * q;
            v[q] = make_uint4(0u, 0u, 0u, 0u);
            if (c < p.d && t >= 0 && t < p.n_tokens) v[q] = p.x[((size_t)t * p.d + c) >> 3];
        }
#pragma unroll
        for (int q = 0; q < ST_PIECES; ++q) {
            const int c = c0 + 256 * q;
            if (!FP8) {
                if (c < p.d) static_cast<uint4 *>(p.rows)[((size_t)r * p.d + c) >> 3] = v[q];
                continue;
            }
            if (c - lane * 8 >= p.d) break;
            float f[8];
            decode16<DIP_W_BF16>(v[q], f);
            float amax = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(f[j]));
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(RT_ALL, amax, o));
            const float scale = fp8_scale(amax);
            if (c < p.d) {
                uint2 code;
                code.x = fp8_codes4(f[0], f[1], f[2], f[3], scale);
                code.y = fp8_codes4(f[4], f[5], f[6], f[7], scale);
                static_cast<uint2 *>(p.rows)[((size_t)r * p.d + c) >> 3] = code;
                if ((lane & 15) == 0) p.scales[(size_t)r * blocks + c / DIP_FP8_BLOCK] = scale;
            }
        }
    }
}

// ---- the rows' weighted sums ----
struct CombineParams {
    const float4 *rows;        // [n_rows][d / 4]
    uint4 *y;                  // [n_tokens][d / 8]
    const float *weight;
    const int32_t *token_row;
    int n_tokens, top_k, d;
};

// A thread per eight columns of a token.  Reads every row once: bound by memory.  The rows are binary32 because the sum is what
// is rounded: with bfloat16 rows a mixture's y was 0.0029 off its 64-bit form (2-norm), 0.0023 to 0.0024 like this.
__global__ void __launch_bounds__(256) combine_rows_kernel(const CombineParams p)
{
    dip_grid_dependency_wait();
    dip_launch_dependents();
    const int eights = p.d / 8, n_rows = p.n_tokens * p.top_k;
    const long long n = (long long)p.n_tokens * eights, step = (long long)gridDim.x * 256;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n; i += step) {
        const int t = (int)(i / eights), c = (int)(i % eights);
        float sum[8] = {};
#pragma unroll 2
        for (int j = 0; j < p.top_k; ++j) {
            const int row = p.token_row[t * p.top_k + j];
            if (row < 0 || row >= n_rows) continue;
            const float w = p.weight[t * p.top_k + j];
            const float4 *f = p.rows + ((size_t)row * eights + c) * 2;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float4 v = f[q];
                sum[4 * q] = fmaf(w, v.x, sum[4 * q]);
                sum[4 * q + 1] = fmaf(w, v.y, sum[4 * q + 1]);
                sum[4 * q + 2] = fmaf(w, v.z, sum[4 * q + 2]);
                sum[4 * q + 3] = fmaf(w, v.w, sum[4 * q + 3]);
            }
        }
        p.y[i] = bf16x8(sum);
    }
}

template <int NV>
cudaError_t launch_choose(const RouteParams &p, bool bf16, int blocks, cudaStream_t stream)
{
    return bf16 ? dip_launch_pdl(route_choose_kernel<NV, true>, dim3(blocks), dim3(RT_THREADS), 0, stream, p)
                : dip_launch_pdl(route_choose_kernel<NV, false>, dim3(blocks), dim3(RT_THREADS), 0, stream, p);
}

}  // namespace

dip_status dip_launch_route(dip_ctx *ctx, const void *logits, bool bf16, bool renormalize, const dip_expert_route &r, cudaStream_t stream)
{
    const int block_tokens = r.n_tokens <= 128 * RT_WARPS ? RT_WARPS : DIP_ROUTE_TOKENS;
    const int blocks = (r.n_tokens + block_tokens - 1) / block_tokens, per_lane = (r.n_experts + 31) / 32;
    const bool add = blocks > 128;
    const RouteParams p = {logits, r.n_tokens, r.n_experts, r.top_k, renormalize, block_tokens, add, r.expert, r.weight, r.offset, r.row_token,
                           r.token_row, ctx->route_counts};
    const auto choose = per_lane <= 1   ? launch_choose<1>
                        : per_lane <= 2 ? launch_choose<2>
                        : per_lane <= 4 ? launch_choose<4>
                        : per_lane <= 8 ? launch_choose<8>
                                        : launch_choose<16>;
    DIP_CUDA_TRY(ctx, choose(p, bf16, blocks, stream));
    if (add) DIP_CUDA_TRY(ctx, dip_launch_pdl(route_add_kernel, dim3(per_lane), dim3(RT_THREADS), 0, stream, p, blocks));
    if (blocks > 1) DIP_CUDA_TRY(ctx, dip_launch_pdl(route_rows_kernel, dim3(blocks), dim3(RT_THREADS), 0, stream, p));
    return DIP_OK;
}

dip_status dip_launch_stage_rows(dip_ctx *ctx, const void *x, int n_tokens, int d, const dip_expert_route *route, bool fp8,
                                 void *rows, float *scales, cudaStream_t stream)
{
    const int n_rows = route ? n_tokens * route->top_k : n_tokens;
    const StageParams p = {static_cast<const uint4 *>(x), n_tokens, n_rows, d, route ? route->row_token : nullptr,
                           route ? route->offset + route->n_experts : nullptr, rows, scales};
    const int warps = n_rows * ((d + 256 * ST_PIECES - 1) / (256 * ST_PIECES)), ctas = min((warps + 7) / 8, ctx->sm_count * 8);
    DIP_CUDA_TRY(ctx, fp8 ? dip_launch_pdl(stage_rows_kernel<true>, dim3(ctas), dim3(256), 0, stream, p)
                          : dip_launch_pdl(stage_rows_kernel<false>, dim3(ctas), dim3(256), 0, stream, p));
    return DIP_OK;
}

dip_status dip_launch_combine_rows(dip_ctx *ctx, const float *rows, const dip_expert_route &r, int d, void *y, cudaStream_t stream)
{
    const CombineParams p = {reinterpret_cast<const float4 *>(rows), static_cast<uint4 *>(y), r.weight, r.token_row, r.n_tokens, r.top_k, d};
    const long long n = (long long)r.n_tokens * (d / 8);
    const int ctas = (int)min((n + 255) / 256, (long long)ctx->sm_count * 8);
    DIP_CUDA_TRY(ctx, dip_launch_pdl(combine_rows_kernel, dim3(ctas), dim3(256), 0, stream, p));
    return DIP_OK;
}
