// Products of groups of rows, a group per expert: y[r] = W[e(r)] rows[r], and h = silu(Wg rows) * (Wu rows).
// Simple form: a block has 16 rows of one expert and 128 outputs, and goes through the input in chunks of 32.
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "common.cuh"
#include "float8.cuh"
#include "gemv_common.cuh"

namespace {

constexpr int GP_ROWS = 16, GP_COLS = 128, GP_K = 32, GP_THREADS = 256;

struct GroupedParams {
    const void *w, *up, *rows;
    const float *w_scales, *up_scales, *row_scales;
    int n_experts, d_out, d_in, n_rows;
    const int32_t *offset;
    void *out;
    float *out_scales;
    int out_f32;
};

template <bool FP8>
__device__ __forceinline__ float grouped_value(const void *p, size_t i)
{
    if (FP8) return (float)static_cast<const __nv_fp8_e4m3 *>(p)[i];
    return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

template <bool FP8, bool GATED>
__global__ void __launch_bounds__(GP_THREADS) grouped_simple_kernel(const GroupedParams p)
{
    __shared__ float sx[GP_ROWS][GP_K + 1], sw[GP_COLS][GP_K + 1], su[GATED ? GP_COLS : 1][GP_K + 1];
    __shared__ float amax[GP_ROWS][16];
    dip_grid_dependency_wait();
    dip_launch_dependents();
    const int tid = threadIdx.x, r = tid >> 4, c = tid & 15, o0 = blockIdx.x * GP_COLS;
    const int kb = (p.d_in + 127) / 128, ob = (p.d_out + 127) / 128;
    for (int e = 0, tile = 0, last = 0; e < p.n_experts; ++e) {
        const int r0 = p.offset ? max(last, min(p.offset[e], p.n_rows)) : 0, r1 = p.offset ? min(p.offset[e + 1], p.n_rows) : p.n_rows;
        last = max(r0, r1);
        for (int m = r0; m < r1; m += GP_ROWS, ++tile) {
            if (tile % gridDim.y != blockIdx.y) continue;
            float a[8] = {}, b[8] = {};
            for (int k0 = 0; k0 < p.d_in; k0 += GP_K) {
                __syncthreads();
                for (int i = tid; i < GP_ROWS * GP_K; i += GP_THREADS) {
                    const int row = m + i / GP_K, k = k0 + i % GP_K;
                    float v = row < r1 ? grouped_value<FP8>(p.rows, (size_t)row * p.d_in + k) : 0.f;
                    if (FP8 && row < r1) v *= p.row_scales[(size_t)row * kb + k / 128];
                    sx[i / GP_K][i % GP_K] = v;
                }
                for (int i = tid; i < GP_COLS * GP_K; i += GP_THREADS) {
                    const int o = o0 + i / GP_K, k = k0 + i % GP_K;
                    const size_t at = ((size_t)e * p.d_out + o) * p.d_in + k, sc = ((size_t)e * ob + o / 128) * kb + k / 128;
                    float v = 0.f, u = 0.f;
                    if (o < p.d_out) {
                        v = grouped_value<FP8>(p.w, at) * (FP8 ? p.w_scales[sc] : 1.f);
                        if (GATED) u = grouped_value<FP8>(p.up, at) * (FP8 ? p.up_scales[sc] : 1.f);
                    }
                    sw[i / GP_K][i % GP_K] = v;
                    if (GATED) su[i / GP_K][i % GP_K] = u;
                }
                __syncthreads();
                for (int k = 0; k < GP_K; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        a[j] = fmaf(sx[r][k], sw[c + 16 * j][k], a[j]);
                        if (GATED) b[j] = fmaf(sx[r][k], su[c + 16 * j][k], b[j]);
                    }
            }
            const int row = m + r;
            float scale = 1.f;
            if (GATED) {
                float most = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    a[j] = silu_f32(a[j]) * b[j];
                    if (o0 + c + 16 * j < p.d_out) most = fmaxf(most, fabsf(a[j]));
                }
                if (FP8) {
                    amax[r][c] = most;
                    __syncthreads();
                    for (int i = 0; i < 16; ++i) most = fmaxf(most, amax[r][i]);
                    scale = fp8_scale(most);
                    if (row < r1 && c == 0) p.out_scales[(size_t)row * ob + blockIdx.x] = scale;
                }
            }
            if (row >= r1) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int o = o0 + c + 16 * j;
                if (o >= p.d_out) continue;
                const size_t at = (size_t)row * p.d_out + o;
                if (GATED && FP8) static_cast<uint8_t *>(p.out)[at] = (uint8_t)fp8_codes4(a[j], 0.f, 0.f, 0.f, scale);
                else if (p.out_f32) static_cast<float *>(p.out)[at] = a[j];
                else static_cast<__nv_bfloat16 *>(p.out)[at] = __float2bfloat16_rn(a[j]);
            }
        }
    }
}

}  // namespace

dip_status dip_launch_grouped(dip_ctx *ctx, const dip_grouped_matrix &w, const dip_grouped_matrix *up, const void *rows,
                              const float *row_scales, int n_rows, const int32_t *offset, void *out, bool out_f32, float *out_scales,
                              cudaStream_t stream)
{
    const bool fp8 = w.wtype == DIP_W_FP8_B128;
    const GroupedParams p = {w.values, up ? up->values : nullptr, rows, w.scales, up ? up->scales : nullptr, row_scales, w.n_experts,
                             w.d_out, w.d_in, n_rows, offset, out, out_scales, out_f32};
    const dim3 grid((w.d_out + GP_COLS - 1) / GP_COLS, min(64, (n_rows + GP_ROWS - 1) / GP_ROWS + w.n_experts)), block(GP_THREADS);
    const auto kernel = fp8 ? (up ? grouped_simple_kernel<true, true> : grouped_simple_kernel<true, false>)
                            : (up ? grouped_simple_kernel<false, true> : grouped_simple_kernel<false, false>);
    DIP_CUDA_TRY(ctx, dip_launch_pdl(kernel, grid, block, 0, stream, p));
    return DIP_OK;
}
