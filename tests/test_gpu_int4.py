"""Products with 4-bit weights and group scales, their gate/up form and the block of them against 64-bit forms."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2412_01380_b200 as dip
import expert_util as eu
import int4_util as iu

pytestmark = pytest.mark.gpu


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


def rows_of(g, n, d):
    return torch.randn((n, d), generator=g, device="cuda").bfloat16()


GROUPS = {
    "one": [1], "two_of_8": [0, 1, 0, 0, 0, 1, 0, 0], "ragged": [5, 0, 130, 1, 0, 64, 33, 0], "first_empty": [0, 0, 3],
    "tile_edges": [128, 127, 129, 256, 1], "small_edges": [8, 7, 9, 16, 17, 15], "none": [0, 0, 0], "many": [3] * 70,
}
# few rows per expert, some, and many: one of them a tile and a row more, or a row short of one
LOADS = {"few": [3, 0, 7], "few_uneven": [130, 0, 3, 0, 0, 1, 0, 0, 0, 0, 0, 2], "more": [1, 24, 0, 25, 2], "some": [70, 0, 90],
         "some_uneven": [129, 1, 30], "many": [400, 0, 250], "many_uneven": [256, 255, 513, 1, 0, 700]}


def check_product(ctx, counts, d_in, d_out, dtype=torch.bfloat16, extra=0, dense=False, seed=0):
    g, n = gen_of(seed), sum(counts) + extra
    w, x = iu.matrix(g, len(counts), d_out, d_in), rows_of(g, max(n, 1), d_in)
    offset = None if dense else eu.offsets(counts)
    y = torch.full((max(n, 1) + 3, d_out), math.nan, device="cuda", dtype=dtype)
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), dip.Rows.of(x), y, offset=offset)
    want, bound = iu.product64(*w, x, offset)
    used = n - extra
    assert torch.isnan(y[used:]).all()                             # rows behind the last group stay as they were
    eu.assert_within(y[:used], want[:used], eu.rounded(want, bound, dtype)[:used], "y")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", list(GROUPS))
def test_product_groups(ctx, name, dtype):
    check_product(ctx, GROUPS[name], 288, 416, dtype, extra=4)


@pytest.mark.parametrize("d_in,d_out", [(32, 32), (64, 256), (96, 1056), (128, 64), (1024, 2816), (2080, 160), (4096, 128), (14336, 96)])
@pytest.mark.parametrize("counts", [[3, 0, 17], [60, 0, 200]])
def test_product_sizes(ctx, d_in, d_out, counts):
    check_product(ctx, counts, d_in, d_out, seed=d_in)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", list(LOADS))
@pytest.mark.parametrize("d_in,d_out", [(8192, 352), (1056, 1184)])
def test_product_loads(ctx, name, d_in, d_out, dtype):
    """Long inputs are cut along K: the tiles' parts meet."""
    check_product(ctx, LOADS[name], d_in, d_out, dtype, extra=2)


def test_more_tiles_than_fit_at_once(ctx):
    check_product(ctx, [500, 20, 900, 0, 130], 160, 5216)
    check_product(ctx, [1, 2, 0, 1] * 16, 96, 5120)


@pytest.mark.parametrize("rows", [1, 2, 4, 8, 9, 16, 17, 31, 33, 128, 200, 1000])
def test_dense_product(ctx, rows):
    check_product(ctx, [rows], 1280, 608, dense=True, seed=rows)


@pytest.mark.parametrize("rows", [1, 9, 40, 150])
@pytest.mark.parametrize("d_in,d_out", [(32768, 64), (64, 32768), (256, 102432), (32, 262144)])
def test_the_widest(ctx, rows, d_in, d_out):
    """The longest rows, and heads: more outputs than any input may have."""
    check_product(ctx, [rows], d_in, d_out, torch.float32, dense=True, seed=rows)


@pytest.mark.parametrize("experts,rows,d_in,d_out", [(512, 600, 96, 64), (512, 9000, 64, 96), (300, 40, 4096, 32), (3, 65536, 64, 64)])
def test_the_most_experts_and_rows(ctx, experts, rows, d_in, d_out):
    g = gen_of(8)
    e = torch.randint(0, experts, (rows,), generator=g, device="cuda").sort().values.int()
    check_product(ctx, torch.bincount(e.long(), minlength=experts).tolist(), d_in, d_out, torch.float32, extra=1, seed=experts)


def test_two_graphs_of_one_context(ctx):
    """They share its workspace, with tiles that are cut in both, and run one after the other."""
    g = gen_of(15)
    m = [dip.GroupedMatrix(*iu.matrix(g, 1, 416, 8192)) for _ in range(2)]
    x = [dip.Rows.of(rows_of(g, n, 8192)) for n in (5, 150)]
    y = [torch.zeros((r.n_rows, 416), device="cuda") for r in x]
    graphs = []
    for i in range(2):
        dip.dip_grouped_product(ctx, m[i], x[i], y[i])
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            dip.dip_grouped_product(ctx, m[i], x[i], y[i])
    want = [v.clone() for v in y]
    for i in (0, 1, 1, 0, 1):
        y[i].zero_()
        graphs[i].replay()
    torch.cuda.synchronize()
    assert torch.equal(y[0], want[0]) and torch.equal(y[1], want[1])


@pytest.mark.parametrize("rows", [2, 12, 150])
def test_large_and_small_inputs(ctx, rows):
    """Rows of very large and of very small values, side by side: products are exact and the sums' bound holds for each row."""
    g = gen_of(9)
    w = iu.matrix(g, 1, 96, 640)
    x = (torch.randn((rows, 640), generator=g, device="cuda") * torch.exp2(torch.linspace(-95, 95, rows, device="cuda"))[:, None]).bfloat16()
    y = torch.zeros((rows, 96), device="cuda")
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), dip.Rows.of(x), y)
    want, bound = iu.product64(*w, x)
    eu.assert_within(y, want, eu.rounded(want, bound, torch.float32), "y")


def test_every_code_and_scale(ctx):
    """One input at a time: y is (code - 8) * scale * x exactly, for every code, and scales that are negative, subnormal, zero or large."""
    g = gen_of(3)
    d_in, d_out = 256, 64
    codes = torch.arange(d_out * d_in // 2, device="cuda").to(torch.uint8).view(1, d_out, d_in // 2)
    scales = torch.tensor([1.0, -2.0, 2.0 ** -24, 3 * 2.0 ** -20, 0.0, 65504.0, -0.333], device="cuda").half()[
        torch.randint(0, 7, (1, 2, d_out), generator=g, device="cuda")]
    x = torch.diag(torch.exp2(torch.randint(-20, 20, (d_in,), generator=g, device="cuda").float())).bfloat16()
    for rows in (1, 9, 256):
        for first in range(0, d_in, rows if rows > 9 else 37):
            part = x[first:first + rows].contiguous()
            y = torch.full((part.shape[0], d_out), math.nan, device="cuda")
            dip.dip_grouped_product(ctx, dip.GroupedMatrix(codes, scales), dip.Rows.of(part), y)
            want = part.double() @ iu.weights64(codes, scales, 0).t()
            assert torch.equal(y.double(), want)


@pytest.mark.parametrize("per", [10, 150])
def test_offsets_are_cut_off(ctx, per):
    """What the offsets name beyond the rows there are is not read or written."""
    g, n = gen_of(5), 4 * per
    w, x = iu.matrix(g, 4, 64, 160), rows_of(g, n, 160)
    offset = torch.tensor([-3, per, per, per - 1, 100 * per], dtype=torch.int32, device="cuda")     # (an expert of less than no rows)
    y = torch.full((n + 20, 64), math.nan, device="cuda", dtype=torch.bfloat16)
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), dip.Rows.of(x), y, offset=offset)
    want, bound = iu.product64(*w, x, offset)
    eu.assert_within(y[:n], want, eu.rounded(want, bound, torch.bfloat16), "y")
    assert torch.isnan(y[n:]).all()


@pytest.mark.parametrize("per", [4, 40, 150])
def test_a_value_that_is_not_finite_stays_in_its_row(ctx, per):
    g = gen_of(6)
    w, x = iu.matrix(g, 2, 96, 320), rows_of(g, 2 * per, 320)
    x[2, 300], x[per + 1, 0] = math.nan, math.inf
    y = torch.zeros((2 * per, 96), device="cuda", dtype=torch.bfloat16)
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), dip.Rows.of(x), y, offset=eu.offsets([per, per]))
    bad = ~torch.isfinite(y)
    # (an infinite x times a code of 8 is NaN, times any other infinite)
    assert bad[2].all() and bad[per + 1].all() and int(bad.any(dim=1).sum()) == 2


@pytest.mark.parametrize("rows", [3, 40, 150])
def test_a_scale_that_is_not_finite_stays_in_its_output(ctx, rows):
    g = gen_of(7)
    codes, scales = iu.matrix(g, 1, 160, 320)
    scales[0, 2, 5], scales[0, 0, 70] = math.nan, math.inf
    y = torch.zeros((rows, 160), device="cuda", dtype=torch.bfloat16)
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(codes, scales), dip.Rows.of(rows_of(g, rows, 320)), y)
    bad = ~torch.isfinite(y)
    assert bad[:, 5].all() and bad[:, 70].all() and int(bad.any(dim=0).sum()) == 2


# ---- gate and up -------------------------------------------------------------------------------------------------------
def check_gate_up(ctx, counts, d_in, d_out, dense=False, seed=0):
    g, n = gen_of(seed), sum(counts)
    gate, up = (iu.matrix(g, len(counts), d_out, d_in) for _ in range(2))
    x = rows_of(g, n, d_in)
    offset = None if dense else eu.offsets(counts)
    h = dip.Rows(n + 2, d_out, dip.W_BF16, "cuda")
    h.values.fill_(55.0)
    dip.dip_grouped_gate_up(ctx, dip.GroupedMatrix(*gate), dip.GroupedMatrix(*up), dip.Rows.of(x), h, offset=offset)
    assert h.n_rows == n and (h.values[n:] == 55.0).all()
    want, bound = iu.gated64(gate, up, x, offset)
    eu.assert_within(h.values[:n], want, eu.rounded(want, bound, torch.bfloat16), "h")


@pytest.mark.parametrize("name", [n for n in GROUPS if n != "none"])
def test_gate_up_groups(ctx, name):
    check_gate_up(ctx, GROUPS[name], 224, 352)


@pytest.mark.parametrize("d_in,d_out", [(32, 32), (64, 96), (1056, 128), (4096, 160), (256, 2816), (128, 32768)])
@pytest.mark.parametrize("counts", [[2, 0, 40], [70, 0, 130]])
def test_gate_up_sizes(ctx, d_in, d_out, counts):
    check_gate_up(ctx, counts, d_in, d_out, seed=d_out)


@pytest.mark.parametrize("name", list(LOADS))
@pytest.mark.parametrize("d_in,d_out", [(8192, 160), (288, 1440)])
def test_gate_up_loads(ctx, name, d_in, d_out):
    check_gate_up(ctx, LOADS[name], d_in, d_out)


@pytest.mark.parametrize("rows", [1, 8, 65, 300])
def test_dense_gate_up(ctx, rows):
    check_gate_up(ctx, [rows], 640, 512, dense=True, seed=rows)


# ---- the block as a whole ----------------------------------------------------------------------------------------------
def weights(g, experts, d_model, d_ff):
    gate, up = (iu.matrix(g, experts, d_ff, d_model) for _ in range(2))
    down = iu.matrix(g, experts, d_model, d_ff)
    return gate, up, down, dip.ExpertWeights(*(dip.GroupedMatrix(*m) for m in (gate, up, down)))


def steps(ctx, w, x, route):
    """The block by its parts."""
    n = x.shape[0] * (route.top_k if route else 1)
    offset = route.offset if route else None
    rows, h = dip.Rows(n, w.d_model, dip.W_BF16, "cuda"), dip.Rows(n, w.d_ff, dip.W_BF16, "cuda")
    out = torch.zeros((n, w.d_model), device="cuda", dtype=torch.float32 if route else torch.bfloat16)
    dip.dip_stage_rows(ctx, x, rows, route=route)
    dip.dip_grouped_gate_up(ctx, w.gate, w.up, rows, h, offset=offset)
    dip.dip_grouped_product(ctx, w.down, h, out, offset=offset)
    if route is None:
        return out, h, out
    y = torch.zeros((x.shape[0], w.d_model), device="cuda", dtype=torch.bfloat16)
    dip.dip_combine_rows(ctx, out, route, y)
    return y, h, out


@pytest.mark.parametrize("tokens,experts,top_k,d_model,d_ff", [
    (1, 8, 2, 1024, 2816), (2, 4, 1, 160, 96), (16, 64, 8, 256, 192), (77, 5, 5, 288, 416), (333, 60, 6, 512, 352), (1500, 8, 2, 256, 512),
])
def test_mixture(ctx, tokens, experts, top_k, d_model, d_ff):
    g = gen_of(tokens)
    gate, up, down, w = weights(g, experts, d_model, d_ff)
    z = torch.randn((tokens, experts), generator=g, device="cuda")
    if tokens > 4:
        z[3] = -math.inf                                           # a padding token: y = 0
    x = rows_of(g, tokens, d_model)
    r, work = dip.ExpertRoute(tokens, experts, top_k, "cuda"), dip.ExpertWork(tokens, top_k, w, "cuda")
    y = torch.full((tokens, d_model), math.nan, device="cuda", dtype=torch.bfloat16)
    dip.dip_route_experts(ctx, z, r)
    dip.dip_expert_mlp(ctx, w, x, work, y, route=r)
    by_parts, h, out = steps(ctx, w, x, r)
    assert torch.equal(y, by_parts)
    # the last product and the weighted sum on the h that the kernels left; the first product has its own tests
    n = int(r.offset[-1])
    want, bound = iu.product64(*down, h.values, r.offset)
    eu.assert_within(out[:n], want[:n], bound[:n], "out")
    at, there = r.token_row.long().clamp_min(0), (r.token_row >= 0)[:, :, None]
    share = r.weight.double()[:, :, None]
    total = torch.where(there, want[at] * share, 0.0).sum(dim=1)
    off = torch.where(there, (bound[at] + want[at].abs() * 2.0 ** -23 * (top_k + 1)) * share, 0.0).sum(dim=1)
    eu.assert_within(y, total, eu.rounded(total, off, torch.bfloat16), "y")
    if tokens > 4:
        assert (y[3] == 0).all()


@pytest.mark.parametrize("tokens", [1, 19, 260])
def test_dense_block_and_in_place(ctx, tokens):
    g = gen_of(tokens)
    gate, up, down, w = weights(g, 1, 544, 800)
    x = rows_of(g, tokens, 544)
    y = torch.full((tokens, 544), math.nan, device="cuda", dtype=torch.bfloat16)
    work = dip.ExpertWork(tokens, 0, w, "cuda")
    dip.dip_expert_mlp(ctx, w, x, work, y)
    by_parts, h, _ = steps(ctx, w, x, None)
    assert torch.equal(y, by_parts)
    want, bound = iu.product64(*down, h.values)
    eu.assert_within(y, want, eu.rounded(want, bound, torch.bfloat16), "y")
    dip.dip_expert_mlp(ctx, w, x, work, x)                         # y over x
    assert torch.equal(x, y)


def test_a_prompt_and_then_decode_steps_from_the_same_arrays(ctx):
    """A model's use: its prompt goes through the dense block at once, its tokens step by step through the packed one, both made of
    the same codes and scales.  A step that keeps every column is the same block; its h stays binary32."""
    d_model, d_ff, g = 512, 1408, gen_of(16)
    gate, up, down, w = weights(g, 1, d_model, d_ff)
    packed = dip.dip_pack_weights(ctx, dip.W_INT4_G128, d_model, d_ff, *(m[0][0] for m in (gate, up, down)),
                                  *(m[1][0] for m in (gate, up, down)))
    x = rows_of(g, 40, d_model)
    y = torch.zeros_like(x)
    dip.dip_expert_mlp(ctx, w, x, dip.ExpertWork(40, 0, w, "cuda"), y)
    one = torch.zeros_like(x)
    work = dip.ExpertWork(1, 0, w, "cuda")
    decoded = torch.zeros((40, d_model), device="cuda")
    for t in range(40):
        dip.dip_expert_mlp(ctx, w, x[t:t + 1], work, one[t:t + 1])
        dip.dip_mlp_step(ctx, packed, x[t].float(), d_model, d_ff, 1.0, None, None, decoded[t])
    h, dh = iu.gated64(gate, up, x)
    down64 = iu.weights64(*down, 0)
    want, mass = h @ down64.t(), h.abs() @ down64.abs().t()
    # the sums of h and y, half a step of h and half a step of y
    off = dh @ down64.abs().t() + mass * (d_ff + 2 * d_ff / 128) * 2.0 ** -23
    eu.assert_within(y, want, off + mass * 2.0 ** -8 + want.abs() * 2.0 ** -8, "prompt")
    eu.assert_within(one, want, off + mass * 2.0 ** -8 + want.abs() * 2.0 ** -8, "one token at a time")
    # (a packed step has its values as two binary16 each: 2^-22 of the largest, so rather of the sum of all)
    eu.assert_within(decoded, want, off + mass * 2.0 ** -11, "packed steps")


# ---- streams, graphs, repetition ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("tokens", [2, 30, 150])
def test_same_bits_again_on_another_stream_and_from_a_graph(ctx, tokens):
    g = gen_of(11)
    w = weights(g, 8, 416, 672)[3]
    z = torch.randn((tokens, 8), generator=g, device="cuda")
    x = rows_of(g, tokens, 416)
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


@pytest.mark.parametrize("rows", [3, 40, 300])
def test_two_contexts_at_once_and_types_in_turn(ctx, rows):
    """Each context has its own workspace: products whose tiles are cut, side by side on two streams, in turn with bfloat16 ones that
    use the same workspace."""
    g = gen_of(14)
    m = dip.GroupedMatrix(*iu.matrix(g, 1, 416, 8192))
    other_type = dip.GroupedMatrix(eu.matrix(g, False, 1, 416, 8192)[0])
    x = [dip.Rows.of(rows_of(g, rows, 8192)) for _ in range(2)]
    alone = []
    for r in x:
        for w in (m, other_type):
            y = torch.zeros((rows, 416), device="cuda", dtype=torch.bfloat16)
            dip.dip_grouped_product(ctx, w, r, y)
            alone.append(y)
    other = dip.Context(0)
    torch.cuda.synchronize()
    streams, both = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(y) for y in alone]
    for _ in range(20):
        for i, (s, c) in enumerate(zip(streams, (ctx, other))):
            with torch.cuda.stream(s):
                dip.dip_grouped_product(c, m, x[i], both[2 * i])
                dip.dip_grouped_product(c, other_type, x[i], both[2 * i + 1])
    torch.cuda.synchronize()
    assert other.device_status() == dip.DEVICE_OK
    other.close()
    for a, b in zip(alone, both):
        assert torch.equal(a, b)


@pytest.mark.parametrize("rows", [1, 7, 40, 150])
def test_rows_that_the_launch_in_front_writes(ctx, rows):
    """A product starts before the launch that stages its rows is through: new rows in the same buffer, launch after launch, give
    what they give one at a time."""
    g = gen_of(4)
    m = dip.GroupedMatrix(*iu.matrix(g, 1, 608, 1280))
    x = [rows_of(g, rows, 1280) for _ in range(40)]
    staged, want = dip.Rows(rows, 1280, dip.W_BF16, "cuda"), []
    for v in x:
        y = torch.zeros((rows, 608), device="cuda")
        dip.dip_stage_rows(ctx, v, staged)
        torch.cuda.synchronize()
        dip.dip_grouped_product(ctx, m, staged, y)
        torch.cuda.synchronize()
        want.append(y)
    got = [torch.zeros_like(y) for y in want]
    torch.cuda.synchronize()
    for v, y in zip(x, got):
        dip.dip_stage_rows(ctx, v, staged)
        dip.dip_grouped_product(ctx, m, staged, y)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


# ---- refusals that need a context --------------------------------------------------------------------------------------
def test_refused_calls_launch_nothing(ctx):
    g = gen_of(12)
    (codes, scales), x = iu.matrix(g, 2, 64, 96), rows_of(g, 5, 96)
    for values, s in ((codes, None), (codes, scales.float()), (codes, scales[:, :, :32].contiguous()), (codes, scales.transpose(1, 2).contiguous()),
                      (codes, scales.cpu()), (codes[:, :, ::2], scales), (codes.to(torch.int8), scales), (codes.bfloat16(), scales)):
        with pytest.raises(dip.DipError):
            dip.GroupedMatrix(values, s)
    m, rows = dip.GroupedMatrix(codes, scales), dip.Rows.of(x)
    y = torch.zeros((5, 64), device="cuda", dtype=torch.bfloat16)
    o = eu.offsets([2, 3])
    q, s = eu.quantise(x)

    def refused(fn, *args, **kw):
        with pytest.raises(dip.DipError) as e:
            fn(ctx, *args, **kw)
        assert e.value.status == dip.ERR_INVALID_ARG

    refused(dip.dip_grouped_product, m, rows, y)                                         # two experts without offsets
    refused(dip.dip_grouped_product, m, dip.Rows.of(q, s), y, offset=o)                  # 8-bit rows
    refused(dip.dip_grouped_product, m, rows, y[:4], offset=o)
    refused(dip.dip_grouped_product, m, rows, y.half(), offset=o)
    refused(dip.dip_grouped_product, m, rows, scales.view(torch.bfloat16).view(-1)[:64].view(1, 64).expand(5, 64), offset=o)
    flat = torch.zeros(4096, device="cuda", dtype=torch.uint8)
    inside = dip.GroupedMatrix(flat[:2 * 64 * 16].view(2, 64, 16), torch.ones((2, 1, 64), device="cuda", dtype=torch.float16))
    short = dip.Rows.of(rows_of(g, 5, 32))
    refused(dip.dip_grouped_product, inside, short, flat[1536:1536 + 640].view(torch.bfloat16).view(5, 64), offset=o)   # y over codes
    mixed = dip.GroupedMatrix(eu.matrix(g, False, 2, 64, 96)[0])
    h = dip.Rows(5, 64, dip.W_BF16, "cuda")
    refused(dip.dip_grouped_gate_up, m, mixed, rows, h, offset=o)                        # gate and up of two types
    wide = dip.GroupedMatrix(torch.zeros((1, 32800, 16), device="cuda", dtype=torch.uint8),
                             torch.zeros((1, 1, 32800), device="cuda", dtype=torch.float16))
    refused(dip.dip_grouped_gate_up, wide, wide, short, dip.Rows(5, 32800, dip.W_BF16, "cuda"))     # a head has no gate
    for d_out, d_in in ((262176, 32), (48, 32), (64, 48)):
        off = dip.GroupedMatrix(torch.zeros((1, d_out, d_in // 2), device="cuda", dtype=torch.uint8),
                                torch.zeros((1, 1, d_out), device="cuda", dtype=torch.float16))
        refused(dip.dip_grouped_product, off, dip.Rows.of(torch.zeros((1, d_in), device="cuda", dtype=torch.bfloat16)),
                torch.zeros((1, d_out), device="cuda"))
    torch.cuda.synchronize()
    assert (y == 0).all() and (flat == 0).all()
