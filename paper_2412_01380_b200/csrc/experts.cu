// C ABI of the router, the grouped products and the expert block (include/dip.h): argument validation and composition.
#include "common.cuh"

namespace {

bool width_ok(int d) { return d >= 32 && d <= DIP_MAX_D && d % 32 == 0; }

// NULL or misaligned
bool bad(const void *p) { return !p || !dip_aligned16(p); }

bool matrix_ok(const dip_grouped_matrix *w)
{
    if (!w || (w->wtype != DIP_W_BF16 && w->wtype != DIP_W_FP8_B128)) return false;
    if (w->n_experts < 1 || w->n_experts > DIP_MAX_EXPERTS || !width_ok(w->d_out) || !width_ok(w->d_in) || bad(w->values)) return false;
    return w->wtype == DIP_W_FP8_B128 ? !bad(w->scales) : !w->scales;
}

bool route_ok(const dip_expert_route *r)
{
    if (!r || r->n_tokens < 1 || r->n_tokens > DIP_MAX_TOKENS || r->n_experts < 1 || r->n_experts > DIP_MAX_EXPERTS) return false;
    if (r->top_k < 1 || r->top_k > DIP_MAX_TOP_K || r->top_k > r->n_experts) return false;
    return !(bad(r->expert) || bad(r->weight) || bad(r->offset) || bad(r->row_token) || bad(r->token_row));
}

// A float type's rows, and the scales that go with it.
bool rows_ok(int wtype, const void *rows, const float *scales)
{
    return !bad(rows) && (wtype == DIP_W_FP8_B128 ? !bad(scales) : !scales);
}

// What a call reads and what it writes share memory.
bool overlap(const void *a, size_t a_bytes, const void *b, size_t b_bytes)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + b_bytes && y < x + a_bytes;
}

size_t row_bytes(int wtype, int n, int d) { return (size_t)n * d * (wtype == DIP_W_FP8_B128 ? 1 : 2); }

bool n_rows_ok(int n) { return n >= 1 && n <= DIP_MAX_TOKENS * DIP_MAX_TOP_K; }

bool same_shape(const dip_grouped_matrix *a, const dip_grouped_matrix *b)
{
    return a->wtype == b->wtype && a->n_experts == b->n_experts && a->d_out == b->d_out && a->d_in == b->d_in;
}

}  // namespace

extern "C" {

dip_status dip_route_experts(dip_ctx *ctx, const void *logits, int logits_bf16, int renormalize, const dip_expert_route *route,
                             void *stream)
{
    if (!dip_ctx_current(ctx) || bad(logits) || !route_ok(route)) return DIP_ERR_INVALID_ARG;
    return dip_launch_route(ctx, logits, logits_bf16 != 0, renormalize != 0, *route, (cudaStream_t)stream);
}

dip_status dip_stage_rows(dip_ctx *ctx, const void *x, int n_tokens, int d, const dip_expert_route *route, int wtype, void *rows,
                          float *scales, void *stream)
{
    if (!dip_ctx_current(ctx) || bad(x) || n_tokens < 1 || n_tokens > DIP_MAX_TOKENS || !width_ok(d)) return DIP_ERR_INVALID_ARG;
    if ((wtype != DIP_W_BF16 && wtype != DIP_W_FP8_B128) || !rows_ok(wtype, rows, scales)) return DIP_ERR_INVALID_ARG;
    if (route && (!route_ok(route) || route->n_tokens != n_tokens)) return DIP_ERR_INVALID_ARG;
    if (overlap(x, row_bytes(DIP_W_BF16, n_tokens, d), rows, row_bytes(wtype, route ? n_tokens * route->top_k : n_tokens, d)))
        return DIP_ERR_INVALID_ARG;
    return dip_launch_stage_rows(ctx, x, n_tokens, d, route, wtype == DIP_W_FP8_B128, rows, scales, (cudaStream_t)stream);
}

dip_status dip_grouped_product(dip_ctx *ctx, const dip_grouped_matrix *w, const void *rows, const float *row_scales, int n_rows,
                               const int32_t *offset, void *y, int y_f32, void *stream)
{
    if (!dip_ctx_current(ctx) || !matrix_ok(w) || !rows_ok(w->wtype, rows, row_scales) || !n_rows_ok(n_rows) || bad(y))
        return DIP_ERR_INVALID_ARG;
    if (offset ? !dip_aligned16(offset) : w->n_experts != 1) return DIP_ERR_INVALID_ARG;
    if (overlap(rows, row_bytes(w->wtype, n_rows, w->d_in), y, (size_t)n_rows * w->d_out * (y_f32 ? 4 : 2))) return DIP_ERR_INVALID_ARG;
    return dip_launch_grouped(ctx, *w, nullptr, rows, row_scales, n_rows, offset, y, y_f32 != 0, nullptr, (cudaStream_t)stream);
}

dip_status dip_grouped_gate_up(dip_ctx *ctx, const dip_grouped_matrix *gate, const dip_grouped_matrix *up, const void *rows,
                               const float *row_scales, int n_rows, const int32_t *offset, void *h, float *h_scales, void *stream)
{
    if (!dip_ctx_current(ctx) || !matrix_ok(gate) || !matrix_ok(up) || !same_shape(gate, up)) return DIP_ERR_INVALID_ARG;
    if (!rows_ok(gate->wtype, rows, row_scales) || !rows_ok(gate->wtype, h, h_scales) || !n_rows_ok(n_rows)) return DIP_ERR_INVALID_ARG;
    if (offset ? !dip_aligned16(offset) : gate->n_experts != 1) return DIP_ERR_INVALID_ARG;
    if (overlap(rows, row_bytes(gate->wtype, n_rows, gate->d_in), h, row_bytes(gate->wtype, n_rows, gate->d_out))) return DIP_ERR_INVALID_ARG;
    return dip_launch_grouped(ctx, *gate, up, rows, row_scales, n_rows, offset, h, false, h_scales, (cudaStream_t)stream);
}

dip_status dip_combine_rows(dip_ctx *ctx, const float *rows, const dip_expert_route *route, int d, void *y, void *stream)
{
    if (!dip_ctx_current(ctx) || bad(rows) || bad(y) || !route_ok(route) || !width_ok(d)) return DIP_ERR_INVALID_ARG;
    return dip_launch_combine_rows(ctx, rows, *route, d, y, (cudaStream_t)stream);
}

dip_status dip_expert_mlp(dip_ctx *ctx, const dip_grouped_matrix *gate, const dip_grouped_matrix *up, const dip_grouped_matrix *down,
                          const void *x, int n_tokens, const dip_expert_route *route, const dip_expert_work *work, void *y,
                          void *stream)
{
    if (!dip_ctx_current(ctx) || !matrix_ok(gate) || !matrix_ok(up) || !matrix_ok(down) || !same_shape(gate, up) || !work)
        return DIP_ERR_INVALID_ARG;
    if (down->wtype != gate->wtype || down->n_experts != gate->n_experts || down->d_out != gate->d_in || down->d_in != gate->d_out)
        return DIP_ERR_INVALID_ARG;
    if (bad(x) || bad(y) || n_tokens < 1 || n_tokens > DIP_MAX_TOKENS) return DIP_ERR_INVALID_ARG;
    if (route ? !route_ok(route) || route->n_tokens != n_tokens || route->n_experts != gate->n_experts : gate->n_experts != 1)
        return DIP_ERR_INVALID_ARG;
    const int wtype = gate->wtype, d = gate->d_in;
    const bool fp8 = wtype == DIP_W_FP8_B128, staged = fp8 || route;
    if ((staged && !rows_ok(wtype, work->rows, work->row_scales)) || !rows_ok(wtype, work->h, work->h_scales) ||
        (route && bad(work->out)))
        return DIP_ERR_INVALID_ARG;
    const cudaStream_t s = (cudaStream_t)stream;
    const int n_rows = route ? n_tokens * route->top_k : n_tokens;
    const size_t x_bytes = row_bytes(DIP_W_BF16, n_tokens, d), h_bytes = row_bytes(wtype, n_rows, gate->d_out);
    if ((staged && overlap(x, x_bytes, work->rows, row_bytes(wtype, n_rows, d))) ||
        overlap(work->h, h_bytes, staged ? work->rows : x, row_bytes(wtype, n_rows, d)) ||
        overlap(work->h, h_bytes, route ? (const void *)work->out : y, (size_t)n_rows * d * (route ? 4 : 2)))
        return DIP_ERR_INVALID_ARG;
    const int32_t *offset = route ? route->offset : nullptr;
    dip_status st = DIP_OK;
    if (staged && (st = dip_launch_stage_rows(ctx, x, n_tokens, d, route, fp8, work->rows, work->row_scales, s)) != DIP_OK) return st;
    if ((st = dip_launch_grouped(ctx, *gate, up, staged ? work->rows : x, work->row_scales, n_rows, offset, work->h, false,
                                 work->h_scales, s)) != DIP_OK)
        return st;
    if ((st = dip_launch_grouped(ctx, *down, nullptr, work->h, work->h_scales, n_rows, offset,
                                 route ? work->out : y, route != nullptr, nullptr, s)) != DIP_OK)
        return st;
    return route ? dip_launch_combine_rows(ctx, work->out, *route, d, y, s) : DIP_OK;
}

}  // extern "C"
