// C ABI of the router, the grouped products and the expert block (include/dip.h): argument validation and composition.
#include <initializer_list>

#include "common.cuh"

namespace {

bool width_ok(int d) { return d >= 32 && d <= DIP_MAX_D && d % 32 == 0; }

// NULL or misaligned
bool bad(const void *p) { return !p || !dip_aligned16(p); }

// head: one of the widths that only a plain 4-bit product takes
bool matrix_ok(const dip_grouped_matrix *w, bool head = false)
{
    if (!w || (w->wtype != DIP_W_BF16 && w->wtype != DIP_W_FP8_B128 && w->wtype != DIP_W_INT4_G128)) return false;
    const bool out_ok = head && w->wtype == DIP_W_INT4_G128 ? w->d_out >= 32 && w->d_out <= DIP_MAX_OUT && w->d_out % 32 == 0 : width_ok(w->d_out);
    if (w->n_experts < 1 || w->n_experts > DIP_MAX_EXPERTS || !out_ok || !width_ok(w->d_in) || bad(w->values)) return false;
    return w->wtype == DIP_W_BF16 ? !w->scales : !bad(w->scales);
}

bool route_ok(const dip_expert_route *r)
{
    if (!r || r->n_tokens < 1 || r->n_tokens > DIP_MAX_TOKENS || r->n_experts < 1 || r->n_experts > DIP_MAX_EXPERTS) return false;
    if (r->top_k < 1 || r->top_k > DIP_MAX_TOP_K || r->top_k > r->n_experts) return false;
    return !(bad(r->expert) || bad(r->weight) || bad(r->offset) || bad(r->row_token) || bad(r->token_row));
}

// The rows that go with a type of weights (4-bit ones take bfloat16), and their scales.
bool rows_ok(int wtype, const void *rows, const float *scales)
{
    return !bad(rows) && (wtype == DIP_W_FP8_B128 ? !bad(scales) : !scales);
}

// A call's buffer; NULL: it has none.
struct Range {
    const void *p;
    size_t bytes;
};

bool meet(const Range &a, const Range &b)
{
    const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
    return a.p && b.p && x < y + b.bytes && y < x + a.bytes;
}

// Whether what is written shares memory with what is read.
bool over(std::initializer_list<Range> written, std::initializer_list<Range> read)
{
    for (const Range &w : written)
        for (const Range &r : read)
            if (meet(w, r)) return true;
    return false;
}

// The same, or with something else that is written.
bool clash(std::initializer_list<Range> written, std::initializer_list<Range> read)
{
    for (const Range *w = written.begin(); w != written.end(); ++w)
        for (const Range *o = written.begin(); o != w; ++o)
            if (meet(*w, *o)) return true;
    return over(written, read);
}

size_t blocks(int d) { return ((size_t)d + DIP_FP8_BLOCK - 1) / DIP_FP8_BLOCK; }
size_t row_bytes(int wtype, int n, int d) { return (size_t)n * d * (wtype == DIP_W_FP8_B128 ? 1 : 2); }
Range row_scales_of(const float *scales, int n, int d) { return {scales, (size_t)n * blocks(d) * sizeof(float)}; }

Range values_of(const dip_grouped_matrix *w)
{
    if (!w) return {};
    return {w->values, (size_t)w->n_experts * (w->wtype == DIP_W_INT4_G128 ? (size_t)w->d_out * w->d_in / 2 : row_bytes(w->wtype, w->d_out, w->d_in))};
}
Range scales_of(const dip_grouped_matrix *w)
{
    if (!w) return {};
    return {w->scales, (size_t)w->n_experts * blocks(w->d_in) * (w->wtype == DIP_W_INT4_G128 ? (size_t)w->d_out * 2 : blocks(w->d_out) * sizeof(float))};
}

size_t choice_bytes(const dip_expert_route *r) { return r ? (size_t)r->n_tokens * r->top_k * 4 : 0; }
Range offset_of(const int32_t *offset, int n_experts) { return {offset, ((size_t)n_experts + 1) * sizeof(int32_t)}; }

// Of one launch each: its blocks run in any order, so what one of them writes may still be read (or written) by others.
bool stage_clash(const void *x, int n_tokens, int d, const dip_expert_route *r, int wtype, const void *rows, const float *scales)
{
    const int n = r ? n_tokens * r->top_k : n_tokens;
    const size_t c = choice_bytes(r);
    return clash({{rows, row_bytes(wtype, n, d)}, row_scales_of(scales, n, d)},
                 {{x, row_bytes(DIP_W_BF16, n_tokens, d)}, {r ? r->expert : nullptr, c}, {r ? r->weight : nullptr, c},
                  offset_of(r ? r->offset : nullptr, r ? r->n_experts : 0), {r ? r->row_token : nullptr, c}, {r ? r->token_row : nullptr, c}});
}

bool product_clash(const dip_grouped_matrix *w, const dip_grouped_matrix *up, const void *rows, const float *row_scales, int n,
                   const int32_t *offset, const void *out, size_t out_bytes, const float *out_scales)
{
    return clash({{out, out_bytes}, row_scales_of(out_scales, n, w->d_out)},
                 {{rows, row_bytes(w->wtype, n, w->d_in)}, row_scales_of(row_scales, n, w->d_in), values_of(w), scales_of(w),
                  values_of(up), scales_of(up), offset_of(offset, w->n_experts)});
}

bool combine_clash(const float *rows, const dip_expert_route *r, int d, const void *y)
{
    const size_t c = choice_bytes(r);
    return over({{y, row_bytes(DIP_W_BF16, r->n_tokens, d)}},
                {{rows, (size_t)r->n_tokens * r->top_k * d * sizeof(float)}, {r->expert, c}, {r->weight, c}, offset_of(r->offset, r->n_experts),
                 {r->row_token, c}, {r->token_row, c}});
}

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
    const size_t c = choice_bytes(route);
    if (clash({{route->expert, c}, {route->weight, c}, offset_of(route->offset, route->n_experts), {route->row_token, c}, {route->token_row, c}},
              {{logits, (size_t)route->n_tokens * route->n_experts * (logits_bf16 ? 2 : 4)}}))
        return DIP_ERR_INVALID_ARG;
    return dip_launch_route(ctx, logits, logits_bf16 != 0, renormalize != 0, *route, (cudaStream_t)stream);
}

dip_status dip_stage_rows(dip_ctx *ctx, const void *x, int n_tokens, int d, const dip_expert_route *route, int wtype, void *rows,
                          float *scales, void *stream)
{
    if (!dip_ctx_current(ctx) || bad(x) || n_tokens < 1 || n_tokens > DIP_MAX_TOKENS || !width_ok(d)) return DIP_ERR_INVALID_ARG;
    if ((wtype != DIP_W_BF16 && wtype != DIP_W_FP8_B128) || !rows_ok(wtype, rows, scales)) return DIP_ERR_INVALID_ARG;
    if (route && (!route_ok(route) || route->n_tokens != n_tokens)) return DIP_ERR_INVALID_ARG;
    if (stage_clash(x, n_tokens, d, route, wtype, rows, scales)) return DIP_ERR_INVALID_ARG;
    return dip_launch_stage_rows(ctx, x, n_tokens, d, route, wtype == DIP_W_FP8_B128, rows, scales, (cudaStream_t)stream);
}

dip_status dip_grouped_product(dip_ctx *ctx, const dip_grouped_matrix *w, const void *rows, const float *row_scales, int n_rows,
                               const int32_t *offset, void *y, int y_f32, void *stream)
{
    if (!dip_ctx_current(ctx) || !matrix_ok(w, true) || !rows_ok(w->wtype, rows, row_scales) || !n_rows_ok(n_rows) || bad(y))
        return DIP_ERR_INVALID_ARG;
    if (offset ? !dip_aligned16(offset) : w->n_experts != 1) return DIP_ERR_INVALID_ARG;
    if (product_clash(w, nullptr, rows, row_scales, n_rows, offset, y, (size_t)n_rows * w->d_out * (y_f32 ? 4 : 2), nullptr))
        return DIP_ERR_INVALID_ARG;
    return dip_launch_grouped(ctx, *w, nullptr, rows, row_scales, n_rows, offset, y, y_f32 != 0, nullptr, (cudaStream_t)stream);
}

dip_status dip_grouped_gate_up(dip_ctx *ctx, const dip_grouped_matrix *gate, const dip_grouped_matrix *up, const void *rows,
                               const float *row_scales, int n_rows, const int32_t *offset, void *h, float *h_scales, void *stream)
{
    if (!dip_ctx_current(ctx) || !matrix_ok(gate) || !matrix_ok(up) || !same_shape(gate, up)) return DIP_ERR_INVALID_ARG;
    if (!rows_ok(gate->wtype, rows, row_scales) || !rows_ok(gate->wtype, h, h_scales) || !n_rows_ok(n_rows)) return DIP_ERR_INVALID_ARG;
    if (offset ? !dip_aligned16(offset) : gate->n_experts != 1) return DIP_ERR_INVALID_ARG;
    if (product_clash(gate, up, rows, row_scales, n_rows, offset, h, row_bytes(gate->wtype, n_rows, gate->d_out), h_scales))
        return DIP_ERR_INVALID_ARG;
    return dip_launch_grouped(ctx, *gate, up, rows, row_scales, n_rows, offset, h, false, h_scales, (cudaStream_t)stream);
}

dip_status dip_combine_rows(dip_ctx *ctx, const float *rows, const dip_expert_route *route, int d, void *y, void *stream)
{
    if (!dip_ctx_current(ctx) || bad(rows) || bad(y) || !route_ok(route) || !width_ok(d) || combine_clash(rows, route, d, y))
        return DIP_ERR_INVALID_ARG;
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
    const int32_t *offset = route ? route->offset : nullptr;
    // each launch by itself, and what an early one writes with what a later one reads; a buffer that is used up may be written again
    // (y over x, say)
    const void *rows = staged ? work->rows : x, *last = route ? (const void *)work->out : y;
    const float *row_scales = fp8 ? work->row_scales : nullptr;
    const size_t c = choice_bytes(route), y_bytes = row_bytes(DIP_W_BF16, n_tokens, d), last_bytes = (size_t)n_rows * d * (route ? 4 : 2);
    if ((staged && stage_clash(x, n_tokens, d, route, wtype, work->rows, row_scales)) ||
        product_clash(gate, up, rows, row_scales, n_rows, offset, work->h, row_bytes(wtype, n_rows, gate->d_out), work->h_scales) ||
        product_clash(down, nullptr, work->h, work->h_scales, n_rows, offset, last, last_bytes, nullptr) ||
        (route && combine_clash(work->out, route, d, y)) ||
        over({{staged ? work->rows : nullptr, row_bytes(wtype, n_rows, d)}, row_scales_of(row_scales, n_rows, d),
              {work->h, row_bytes(wtype, n_rows, gate->d_out)}, row_scales_of(work->h_scales, n_rows, gate->d_out), {last, last_bytes}, {y, y_bytes}},
             {values_of(gate), scales_of(gate), values_of(up), scales_of(up), values_of(down), scales_of(down),
              {route ? route->expert : nullptr, c}, {route ? route->weight : nullptr, c}, {route ? route->row_token : nullptr, c},
              {route ? route->token_row : nullptr, c}, offset_of(offset, gate->n_experts)}))
        return DIP_ERR_INVALID_ARG;
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
