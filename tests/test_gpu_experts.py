"""Router, grouped products (bfloat16 and 8-bit weights) and the expert block against their 64-bit forms (tests/expert_util.py)."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2412_01380_b200 as dip
import expert_util as eu

pytestmark = pytest.mark.gpu
WTYPES = {"bf16": dip.W_BF16, "fp8": dip.W_FP8_B128}


@pytest.fixture(scope="module")
def ctx():
    c = dip.Context(0)
    yield c
    assert c.device_status() == dip.DEVICE_OK
    c.close()


def gen_of(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def nan_like(shape, dtype):
    return torch.full(shape, math.nan, device="cuda", dtype=dtype)


# ---- router ------------------------------------------------------------------------------------------------------------
def check_route(ctx, logits, top_k, renormalize, route=None):
    tokens, experts = logits.shape
    r = route or dip.ExpertRoute(tokens, experts, top_k, "cuda")
    r.row_token.fill_(-7)
    dip.dip_route_experts(ctx, logits, r, renormalize=renormalize)
    expert, weight, offset, row_token, token_row = eu.route64(logits, top_k, renormalize)
    assert torch.equal(r.expert[:tokens].cpu(), expert)
    assert torch.equal(r.offset.cpu(), offset)
    assert torch.equal(r.token_row[:tokens].cpu(), token_row)
    n = int(offset[-1])
    assert torch.equal(r.row_token[:n].cpu(), row_token)
    assert (r.row_token[n:] == -7).all()                           # rows behind the last group stay as they were
    # exp(v - max) in binary32: the difference is rounded (2^-24 of at most some tens), exp to 2 units, sums of up to 512 parts
    big = logits.float()[torch.isfinite(logits)].abs().max().item() if torch.isfinite(logits).any() else 0.0
    eu.assert_within(r.weight[:tokens].cpu(), weight, weight * (4 * big * 2.0 ** -24 + (experts + 16) * 2.0 ** -24) + 2.0 ** -126, "weight")
    return r


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("tokens,experts,top_k,dtype", [
    (1, 1, 1, "f32"), (1, 64, 8, "f32"), (3, 8, 2, "bf16"), (17, 33, 4, "f32"), (127, 60, 6, "bf16"), (128, 128, 8, "f32"),
    (129, 5, 5, "bf16"), (300, 512, 16, "f32"), (1000, 100, 3, "bf16"), (2049, 256, 1, "f32"),
])
def test_route(ctx, tokens, experts, top_k, dtype, renormalize):
    z = torch.randn((tokens, experts), generator=gen_of(tokens), device="cuda") * 2
    check_route(ctx, z.bfloat16() if dtype == "bf16" else z, top_k, renormalize)


@pytest.mark.parametrize("tokens", [5, 200])
@pytest.mark.parametrize("renormalize", [False, True])
def test_route_closed_experts_and_padding(ctx, tokens, renormalize):
    z = torch.randn((tokens, 24), generator=gen_of(3), device="cuda")
    z[torch.rand(z.shape, generator=gen_of(4), device="cuda") < 0.6] = -math.inf
    z[1] = -math.inf                                               # nothing left
    z[2] = -math.inf
    z[2, 23] = 1.5                                                 # fewer than top_k
    z[3, ::2] = math.nan
    z[4] = torch.finfo(torch.float32).min                          # the lowest finite value is open
    check_route(ctx, z, 4, renormalize)


@pytest.mark.parametrize("renormalize", [False, True])
def test_route_ties_zeros_and_infinities(ctx, renormalize):
    z = torch.zeros((6, 40), device="cuda")
    z[0, 3::4] = -0.0                                              # equal to 0: index order
    z[1] = torch.tensor([1.0, 2.0] * 20)
    z[2, 7], z[2, 30] = math.inf, math.inf
    z[3, 9] = math.inf
    z[4] = -5e4
    z[5, 39] = 1e-30
    check_route(ctx, z, 6, renormalize)


def test_route_all_tokens_padding(ctx):
    r = check_route(ctx, torch.full((150, 8), -math.inf, device="cuda"), 2, True)
    assert int(r.offset[-1]) == 0


def test_route_one_expert_takes_all(ctx):
    z = torch.zeros((700, 16), device="cuda")
    z[:, 5] = 9
    check_route(ctx, z, 1, True)


@pytest.mark.parametrize("tokens,experts,top_k", [(20000, 40, 2), (65536, 8, 1), (16385, 500, 16)])
def test_route_of_many_tokens(ctx, tokens, experts, top_k):
    """Many blocks: against a sort (the token by token form takes minutes)."""
    z = torch.randn((tokens, experts), generator=gen_of(tokens), device="cuda")
    z[::7] = -math.inf
    r = dip.ExpertRoute(tokens, experts, top_k, "cuda")
    dip.dip_route_experts(ctx, z, r)
    expert = torch.argsort(z, dim=1, descending=True, stable=True)[:, :top_k].int()
    expert[::7] = -1
    assert torch.equal(r.expert, expert)
    key = torch.where(expert < 0, experts, expert).flatten().long()
    order = torch.argsort(key, stable=True)
    offset = torch.searchsorted(key[order], torch.arange(experts + 1, device="cuda")).int()
    assert torch.equal(r.offset, offset)
    n = int(offset[-1])
    assert torch.equal(r.row_token[:n], (order // top_k)[:n].int())
    row = torch.empty_like(order).scatter_(0, order, torch.arange(order.numel(), device="cuda"))
    assert torch.equal(r.token_row.flatten(), torch.where(key == experts, -1, row).int())


def test_route_is_used_again_with_fewer_tokens(ctx):
    r = dip.ExpertRoute(300, 12, 3, "cuda")
    z = torch.randn((300, 12), generator=gen_of(8), device="cuda")
    check_route(ctx, z, 3, True, r)
    check_route(ctx, z[:7].contiguous(), 3, True, r)
    assert r.n_tokens == 7


# ---- rows --------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("tokens,d", [(1, 32), (3, 160), (70, 1056), (5, 4096)])
def test_stage_rows_dense(ctx, wtype, tokens, d):
    x = (torch.randn((tokens, d), generator=gen_of(d), device="cuda") * 3).bfloat16()
    x[0, :32] = 0
    rows = dip.Rows(tokens + 2, d, WTYPES[wtype], "cuda")
    rows.values.view(torch.uint8).fill_(99)
    dip.dip_stage_rows(ctx, x, rows)
    assert rows.n_rows == tokens
    assert (rows.values[tokens:].view(torch.uint8) == 99).all()
    if wtype == "bf16":
        assert torch.equal(rows.values[:tokens], x)
    else:
        q, s = eu.quantise(x)
        assert torch.equal(rows.scales[:tokens], s)
        assert torch.equal(rows.values[:tokens].view(torch.uint8), q.view(torch.uint8))


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
def test_stage_rows_of_a_route(ctx, wtype):
    z = torch.randn((37, 10), generator=gen_of(1), device="cuda")
    z[5] = -math.inf
    r = dip.ExpertRoute(37, 10, 3, "cuda")
    dip.dip_route_experts(ctx, z, r)
    x = torch.randn((37, 288), generator=gen_of(2), device="cuda").bfloat16()
    rows = dip.Rows(37 * 3, 288, WTYPES[wtype], "cuda")
    rows.values.view(torch.uint8).fill_(77)
    dip.dip_stage_rows(ctx, x, rows, route=r)
    n = int(r.offset[-1])
    assert n == 36 * 3
    want = x[r.row_token[:n].long()]
    if wtype == "fp8":
        want, s = eu.quantise(want)
        assert torch.equal(rows.scales[:n], s)
    assert torch.equal(rows.values[:n].view(torch.uint8), want.view(torch.uint8))
    assert (rows.values[n:].view(torch.uint8) == 77).all()


def test_stage_rows_extremes(ctx):
    x = torch.zeros((6, 256), device="cuda", dtype=torch.bfloat16)
    x[1, :] = torch.finfo(torch.bfloat16).max
    x[2, 0] = 2.0 ** -133                                          # the smallest bfloat16: 2^-7 of the smallest scale, a code
    x[3, 7] = math.nan
    x[4, 200] = -math.inf
    x[5, ::2] = 1e-30
    rows = dip.Rows(6, 256, dip.W_FP8_B128, "cuda")
    dip.dip_stage_rows(ctx, x, rows)
    v = eu.values64(rows.values, rows.scales)
    assert (v[0] == 0).all() and torch.equal(v[2], x[2].double())
    for r in (1, 5):
        eu.assert_within(v[r], x[r].double(), x[r].double().abs() * (2.0 ** -4 + 2.0 ** -20), "row %d" % r)
    assert torch.isnan(v[3]).sum() == 1 and torch.isnan(v[3, 7])
    assert torch.isnan(v[4, 200])


# ---- grouped products --------------------------------------------------------------------------------------------------
GROUPS = {
    "one": [1], "two_of_8": [0, 1, 0, 0, 0, 1, 0, 0], "ragged": [5, 0, 130, 1, 0, 64, 33, 0], "first_empty": [0, 0, 3],
    "tile_edges": [128, 127, 129, 256, 1], "none": [0, 0, 0], "many": [3] * 70,
}


def check_product(ctx, wtype, counts, d_in, d_out, dtype=torch.bfloat16, extra=0, dense=False, seed=0):
    g = gen_of(seed)
    fp8, experts = wtype == "fp8", len(counts)
    n = sum(counts) + extra
    w = eu.matrix(g, fp8, experts, d_out, d_in)
    x = eu.rows_of(g, fp8, max(n, 1), d_in)
    offset = None if dense else eu.offsets(counts)
    y = nan_like((max(n, 1) + 3, d_out), dtype)
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), dip.Rows.of(*x), y, offset=offset)
    want, bound = eu.product64(*w, eu.values64(*x), offset)
    used = n - extra
    assert torch.isnan(y[used:]).all()                             # rows behind the last group stay as they were
    eu.assert_within(y[:used], want[:used], eu.rounded(want, bound, dtype)[:used], "y")
    return y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("name", list(GROUPS))
def test_grouped_product_groups(ctx, wtype, name, dtype):
    check_product(ctx, wtype, GROUPS[name], 288, 416, dtype, extra=4)


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d_in,d_out", [(32, 32), (64, 256), (96, 1056), (1024, 2816), (2080, 160), (4096, 128), (14336, 96)])
def test_grouped_product_sizes(ctx, wtype, d_in, d_out):
    check_product(ctx, wtype, [3, 0, 17], d_in, d_out, seed=d_in)


# few rows per expert, some, and many: one of them a tile and a row more, or a row short of one
LOADS = {"few": [3, 0, 17], "few_uneven": [130, 0, 3, 0, 0, 1, 0, 0, 0, 0, 0, 2], "more_than_a_tile_of_few": [1, 64, 0, 65, 2], "some": [70, 0, 90], "some_uneven": [129, 1, 30],
         "many": [400, 0, 250], "many_uneven": [256, 255, 513, 1, 0, 700]}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("name", list(LOADS))
@pytest.mark.parametrize("d_in,d_out", [(8192, 352), (1056, 1184)])
def test_grouped_product_loads(ctx, wtype, name, d_in, d_out, dtype):
    """Long inputs are cut along K: the tiles' parts meet."""
    check_product(ctx, wtype, LOADS[name], d_in, d_out, dtype, extra=2)


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
def test_more_tiles_than_fit_at_once(ctx, wtype):
    check_product(ctx, wtype, [500, 20, 900, 0, 130], 160, 5216)
    check_product(ctx, wtype, [1, 2, 0, 1] * 16, 96, 5120)


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("rows", [1, 2, 31, 33, 200, 1000])
def test_dense_product(ctx, wtype, rows):
    check_product(ctx, wtype, [rows], 1280, 608, dense=True, seed=rows)


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
def test_grouped_product_offsets_are_cut_off(ctx, wtype):
    """What the offsets name beyond the rows there are is not read or written."""
    g, fp8 = gen_of(5), wtype == "fp8"
    w, x = eu.matrix(g, fp8, 4, 64, 160), eu.rows_of(g, fp8, 40, 160)
    offset = torch.tensor([-3, 10, 10, 9, 4000], dtype=torch.int32, device="cuda")     # (9: an expert of less than no rows)
    y = nan_like((60, 64), torch.bfloat16)
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), dip.Rows.of(*x), y, offset=offset)
    want, bound = eu.product64(*w, eu.values64(*x), offset)
    eu.assert_within(y[:40], want, eu.rounded(want, bound, torch.bfloat16), "y")
    assert torch.isnan(y[40:]).all()


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
def test_a_value_that_is_not_finite_stays_in_its_row(ctx, wtype):
    g, fp8 = gen_of(6), wtype == "fp8"
    w = eu.matrix(g, fp8, 2, 96, 320)
    x = torch.randn((9, 320), generator=g, device="cuda").bfloat16()
    x[2, 300], x[6, 0] = math.nan, math.inf
    rows = dip.Rows(9, 320, WTYPES[wtype], "cuda")
    dip.dip_stage_rows(ctx, x, rows)
    y = torch.zeros((9, 96), device="cuda", dtype=torch.bfloat16)
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), rows, y, offset=eu.offsets([4, 5]))
    bad = ~torch.isfinite(y)
    assert bad[2].all() and bad[6].all() and int(bad.any(dim=1).sum()) == 2


def check_gate_up(ctx, wtype, counts, d_in, d_out, dense=False, seed=0):
    g, fp8 = gen_of(seed), wtype == "fp8"
    n = sum(counts)
    gate, up = (eu.matrix(g, fp8, len(counts), d_out, d_in) for _ in range(2))
    x = eu.rows_of(g, fp8, n, d_in)
    offset = None if dense else eu.offsets(counts)
    h = dip.Rows(n + 2, d_out, WTYPES[wtype], "cuda")
    h.values.view(torch.uint8).fill_(55)
    dip.dip_grouped_gate_up(ctx, dip.GroupedMatrix(*gate), dip.GroupedMatrix(*up), dip.Rows.of(*x), h, offset=offset)
    assert h.n_rows == n and (h.values[n:].view(torch.uint8) == 55).all()
    want, bound = eu.gated64(gate, up, eu.values64(*x), offset)
    if not fp8:
        eu.assert_within(h.values[:n], want, eu.rounded(want, bound, torch.bfloat16), "h")
        return h
    # the scale is that of the largest value to within the sums' error; a code is off by half a step (normal or subnormal)
    pad = lambda v: torch.nn.functional.pad(v, (0, -d_out % eu.BLOCK)).view(n, -1, eu.BLOCK)  # noqa: E731
    scale = pad(want.abs()).amax(dim=2) / 448
    eu.assert_within(h.scales[:n], scale.clamp_min(eu.TINY), pad(bound).amax(dim=2) / 448 + scale * 2.0 ** -22, "scale")
    per = h.scales[:n].double().repeat_interleave(eu.BLOCK, dim=1)[:, :d_out]
    eu.assert_within(eu.values64(h.values[:n], h.scales[:n]), want, bound + 2.0 ** -4 * (want.abs() + bound) + per * 2.0 ** -10 +
                     want.abs() * 2.0 ** -20, "h")
    return h


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("name", [n for n in GROUPS if n != "none"])
def test_gate_up_groups(ctx, wtype, name):
    check_gate_up(ctx, wtype, GROUPS[name], 224, 352)


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d_in,d_out", [(32, 32), (64, 96), (1056, 128), (4096, 160), (256, 2816)])
def test_gate_up_sizes(ctx, wtype, d_in, d_out):
    check_gate_up(ctx, wtype, [2, 0, 40], d_in, d_out, seed=d_out)


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("name", list(LOADS))
@pytest.mark.parametrize("d_in,d_out", [(8192, 160), (288, 1440)])
def test_gate_up_loads(ctx, wtype, name, d_in, d_out):
    check_gate_up(ctx, wtype, LOADS[name], d_in, d_out)


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("rows", [1, 65, 300])
def test_dense_gate_up(ctx, wtype, rows):
    check_gate_up(ctx, wtype, [rows], 640, 512, dense=True, seed=rows)


# ---- the block as a whole ----------------------------------------------------------------------------------------------
def weights(g, fp8, experts, d_model, d_ff):
    gate, up = (eu.matrix(g, fp8, experts, d_ff, d_model) for _ in range(2))
    down = eu.matrix(g, fp8, experts, d_model, d_ff)
    return gate, up, down, dip.ExpertWeights(*(dip.GroupedMatrix(*m) for m in (gate, up, down)))


def steps(ctx, w, x, route):
    """The block by its four parts."""
    n = x.shape[0] * (route.top_k if route else 1)
    offset = route.offset if route else None
    rows, h = dip.Rows(n, w.d_model, w.wtype, "cuda"), dip.Rows(n, w.d_ff, w.wtype, "cuda")
    out = torch.zeros((n, w.d_model), device="cuda", dtype=torch.float32 if route else torch.bfloat16)
    y = torch.zeros((x.shape[0], w.d_model), device="cuda", dtype=torch.bfloat16)
    dip.dip_stage_rows(ctx, x, rows, route=route)
    dip.dip_grouped_gate_up(ctx, w.gate, w.up, rows, h, offset=offset)
    dip.dip_grouped_product(ctx, w.down, h, out, offset=offset)
    if route is None:
        return out, h, out
    dip.dip_combine_rows(ctx, out, route, y)
    return y, h, out


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("tokens,experts,top_k,d_model,d_ff", [
    (1, 8, 2, 1024, 2816), (2, 4, 1, 160, 96), (16, 64, 8, 256, 192), (77, 5, 5, 288, 416), (333, 60, 6, 512, 352), (1500, 8, 2, 256, 512),
])
def test_mixture(ctx, wtype, tokens, experts, top_k, d_model, d_ff):
    g, fp8 = gen_of(tokens), wtype == "fp8"
    gate, up, down, w = weights(g, fp8, experts, d_model, d_ff)
    z = torch.randn((tokens, experts), generator=g, device="cuda")
    if tokens > 4:
        z[3] = -math.inf                                           # a padding token: y = 0
    x = torch.randn((tokens, d_model), generator=g, device="cuda").bfloat16()
    r = dip.ExpertRoute(tokens, experts, top_k, "cuda")
    work = dip.ExpertWork(tokens, top_k, w, "cuda")
    y = nan_like((tokens, d_model), torch.bfloat16)
    dip.dip_route_experts(ctx, z, r)
    dip.dip_expert_mlp(ctx, w, x, work, y, route=r)
    by_parts, h, out = steps(ctx, w, x, r)
    assert torch.equal(y, by_parts)
    # the last product and the weighted sum on the h that the kernels left; the first product has its own tests
    n = int(r.offset[-1])
    want, bound = eu.product64(*down, eu.values64(h.values, h.scales), r.offset)
    eu.assert_within(out[:n], want[:n], bound[:n], "out")
    at, there = r.token_row.long().clamp_min(0), (r.token_row >= 0)[:, :, None]
    share = r.weight.double()[:, :, None]
    total = torch.where(there, want[at] * share, 0.0).sum(dim=1)
    off = torch.where(there, (bound[at] + want[at].abs() * 2.0 ** -23 * (top_k + 1)) * share, 0.0).sum(dim=1)
    eu.assert_within(y, total, eu.rounded(total, off, torch.bfloat16), "y")
    if tokens > 4:
        assert (y[3] == 0).all()


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("tokens", [1, 19, 260])
def test_dense_block(ctx, wtype, tokens):
    g, fp8 = gen_of(tokens), wtype == "fp8"
    gate, up, down, w = weights(g, fp8, 1, 544, 800)
    x = torch.randn((tokens, 544), generator=g, device="cuda").bfloat16()
    y = nan_like((tokens, 544), torch.bfloat16)
    dip.dip_expert_mlp(ctx, w, x, dip.ExpertWork(tokens, 0, w, "cuda"), y)
    by_parts, h, _ = steps(ctx, w, x, None)
    assert torch.equal(y, by_parts)
    want, bound = eu.product64(*down, eu.values64(h.values, h.scales))
    eu.assert_within(y, want, eu.rounded(want, bound, torch.bfloat16), "y")


def test_combine_is_the_weighted_sum_in_order(ctx):
    r = dip.ExpertRoute(50, 9, 4, "cuda")
    z = torch.randn((50, 9), generator=gen_of(1), device="cuda")
    z[7], z[8, 1:] = -math.inf, -math.inf
    dip.dip_route_experts(ctx, z, r, renormalize=False)
    rows = torch.randn((200, 96), generator=gen_of(2), device="cuda")
    rows[int(r.offset[-1]):] = math.nan
    y = nan_like((50, 96), torch.bfloat16)
    dip.dip_combine_rows(ctx, rows, r, y)
    parts = torch.where((r.token_row >= 0)[:, :, None], rows.double()[r.token_row.long().clamp_min(0)] * r.weight.double()[:, :, None], 0.0)
    eu.assert_within(y, parts.sum(1), eu.rounded(parts.sum(1), parts.abs().sum(1) * 8 * 2.0 ** -24, torch.bfloat16), "y")
    assert (y[7] == 0).all()


# ---- streams, graphs, repetition ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("tokens", [2, 150])
def test_same_bits_again_on_another_stream_and_from_a_graph(ctx, wtype, tokens):
    g = gen_of(11)
    w = weights(g, wtype == "fp8", 8, 416, 672)[3]
    z = torch.randn((tokens, 8), generator=g, device="cuda")
    x = torch.randn((tokens, 416), generator=g, device="cuda").bfloat16()
    r, work = dip.ExpertRoute(tokens, 8, 2, "cuda"), dip.ExpertWork(tokens, 2, w, "cuda")
    y = torch.zeros((tokens, 416), device="cuda", dtype=torch.bfloat16)

    def call():
        dip.dip_route_experts(ctx, z, r)
        dip.dip_expert_mlp(ctx, w, x, work, y, route=r)

    call()
    first = y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            y.zero_()
            call()
            assert torch.equal(y, first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    # new inputs through the captured call
    z.copy_(torch.randn(z.shape, generator=g, device="cuda"))
    x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    for _ in range(2):
        graph.replay()
    again = y.clone()
    y.zero_()
    call()
    assert torch.equal(y, again) and not torch.equal(y, first)


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
def test_two_contexts_at_once(ctx, wtype):
    """Each context has its own workspace: products whose tiles are cut, side by side on two streams."""
    g = gen_of(14)
    m = dip.GroupedMatrix(*eu.matrix(g, wtype == "fp8", 4, 416, 8192))
    rows = [dip.Rows.of(*eu.rows_of(g, wtype == "fp8", 40, 8192)) for _ in range(2)]
    o = eu.offsets([5, 30, 0, 5])
    alone = []
    for r in rows:
        y = torch.zeros((40, 416), device="cuda", dtype=torch.bfloat16)
        dip.dip_grouped_product(ctx, m, r, y, offset=o)
        alone.append(y)
    other = dip.Context(0)
    torch.cuda.synchronize()
    streams, both = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(y) for y in alone]
    for _ in range(20):
        for s, c, r, y in zip(streams, (ctx, other), rows, both):
            with torch.cuda.stream(s):
                dip.dip_grouped_product(c, m, r, y, offset=o)
    torch.cuda.synchronize()
    assert other.device_status() == dip.DEVICE_OK
    other.close()
    for a, b in zip(alone, both):
        assert torch.equal(a, b)


def test_two_graphs_of_one_context(ctx):
    """They share its workspace and run one after the other."""
    g = gen_of(15)
    w = [weights(g, fp8, 8, 256, 2080)[3] for fp8 in (False, True)]
    x = torch.randn((9, 256), generator=g, device="cuda").bfloat16()
    z = torch.randn((9, 8), generator=g, device="cuda")
    route = [dip.ExpertRoute(9, 8, 3, "cuda") for _ in w]
    work, y = [dip.ExpertWork(9, 3, v, "cuda") for v in w], [torch.zeros_like(x) for _ in w]

    def call(i):
        dip.dip_route_experts(ctx, z, route[i])
        dip.dip_expert_mlp(ctx, w[i], x, work[i], y[i], route=route[i])

    graphs = []
    for i in range(2):
        call(i)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            call(i)
    want = [v.clone() for v in y]
    for i in (0, 1, 1, 0, 1):
        y[i].zero_()
        graphs[i].replay()
    torch.cuda.synchronize()
    assert torch.equal(y[0], want[0]) and torch.equal(y[1], want[1])


def test_a_prompt_and_then_decode_steps(ctx):
    """A model's use: its prompt goes through the dense block at once, its tokens step by step through the packed one, on one
    context.  A step that keeps every column is the same block; its h stays binary32, the dense block's is rounded once."""
    d_model, d_ff, g = 512, 1376, gen_of(16)
    gate, up = (torch.randn((d_ff, d_model), generator=g, device="cuda").mul_(0.05).bfloat16() for _ in range(2))
    down = torch.randn((d_model, d_ff), generator=g, device="cuda").mul_(0.05).bfloat16()
    packed = dip.dip_pack_weights(ctx, dip.W_BF16, d_model, d_ff, gate, up, down)
    w = dip.ExpertWeights(*(dip.GroupedMatrix(m) for m in (gate, up, down)))
    x = torch.randn((40, d_model), generator=g, device="cuda").bfloat16()
    y = torch.zeros_like(x)
    dip.dip_expert_mlp(ctx, w, x, dip.ExpertWork(40, 0, w, "cuda"), y)
    steps = torch.zeros((40, d_model), device="cuda")
    for t in range(0, 40, 8):
        dip.dip_mlp_step(ctx, packed, x[t].float(), d_model, d_ff, 1.0, None, None, steps[t])
        dip.dip_mlp_step(ctx, packed, x[t + 1:t + 8].float(), d_model, d_ff, 1.0, None, None, steps[t + 1:t + 8])
    h = x.double() @ gate.double().t()
    h = h * torch.sigmoid(h) * (x.double() @ up.double().t())
    want = h @ down.double().t()
    mass = h.abs() @ down.double().abs().t()
    # half a step of h, half a step of y, and binary32 sums over d_model and d_ff
    eu.assert_within(y, want, mass * (2.0 ** -8 + 2.0 ** -11) + want.abs() * 2.0 ** -8, "prompt")
    # (a batch stands for each value by two bfloat16: 2^-16)
    eu.assert_within(steps, want, mass * 2.0 ** -11, "steps")
    again = torch.zeros_like(x)
    dip.dip_expert_mlp(ctx, w, x, dip.ExpertWork(40, 0, w, "cuda"), again)
    assert torch.equal(y, again)


# ---- refusals that need a context --------------------------------------------------------------------------------------
def test_refused_calls_launch_nothing(ctx):
    g = gen_of(12)
    w, x = eu.matrix(g, False, 2, 64, 96), eu.rows_of(g, False, 5, 96)
    m, rows = dip.GroupedMatrix(*w), dip.Rows.of(*x)
    y = torch.zeros((5, 64), device="cuda", dtype=torch.bfloat16)
    o = eu.offsets([2, 3])
    bad = [
        dict(),                                                    # two experts without offsets
        dict(offset=o[:2].contiguous()), dict(offset=o.long()), dict(offset=o.cpu()),
        dict(offset=torch.zeros(4, dtype=torch.int32, device="cuda")[1:]),           # 4 bytes off a boundary of 16
    ]
    for kw in bad:
        with pytest.raises(dip.DipError):
            dip.dip_grouped_product(ctx, m, rows, y, **kw)
    for out in (y[:4], y.half(), y.t(), torch.zeros((5, 32), device="cuda", dtype=torch.bfloat16), y.cpu()):
        with pytest.raises(dip.DipError):
            dip.dip_grouped_product(ctx, m, rows, out, offset=o)
    square = dip.GroupedMatrix(eu.matrix(g, False, 1, 96, 96)[0])
    with pytest.raises(dip.DipError):                              # in place: rows that others still read
        dip.dip_grouped_product(ctx, square, rows, rows.values)
    with pytest.raises(dip.DipError):
        dip.dip_stage_rows(ctx, rows.values, rows)
    with pytest.raises(dip.DipError):                              # 48 columns: no multiple of 32
        narrow = dip.GroupedMatrix(torch.zeros((2, 64, 48), device="cuda", dtype=torch.bfloat16))
        dip.dip_grouped_product(ctx, narrow, dip.Rows.of(torch.zeros((5, 48), device="cuda", dtype=torch.bfloat16)), y, offset=o)
    torch.cuda.synchronize()
    assert (y == 0).all()
