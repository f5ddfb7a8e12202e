"""Uses of the router, the grouped products and the expert block at the edge of what a call takes: buffers that share memory,
waits that run out."""
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


def block(g, fp8, experts, d_model, d_ff):
    gate, up = (dip.GroupedMatrix(*eu.matrix(g, fp8, experts, d_ff, d_model)) for _ in range(2))
    return dip.ExpertWeights(gate, up, dip.GroupedMatrix(*eu.matrix(g, fp8, experts, d_model, d_ff)))


def test_calls_that_write_what_they_read_are_refused(ctx):
    g = gen_of(1)
    w = block(g, True, 3, 256, 256)
    rows, h = dip.Rows.of(*eu.rows_of(g, True, 9, 256)), dip.Rows(9, 256, dip.W_FP8_B128, "cuda")
    h.values.view(torch.uint8).fill_(3)
    o, scales = eu.offsets([4, 0, 5]), rows.scales.clone()

    def refused(fn, *args, **kw):
        with pytest.raises(dip.DipError) as e:
            fn(ctx, *args, **kw)
        assert e.value.status == dip.ERR_INVALID_ARG

    # an 8-bit h whose scales, or whose codes, are where the rows' scales are (256 to 256: they have the same shape)
    same = dip.Rows.of(h.values, rows.scales)
    refused(dip.dip_grouped_gate_up, w.gate, w.up, rows, same, offset=o)
    both = torch.zeros(9 * 256 + 64, dtype=torch.uint8, device="cuda")
    codes, their = both[:9 * 256].view(torch.float8_e4m3fn).view(9, 256), both[9 * 256 - 16:9 * 256 + 56].view(torch.float32).view(9, 2)
    refused(dip.dip_grouped_gate_up, w.gate, w.up, dip.Rows.of(rows.values, their), dip.Rows.of(codes, h.scales), offset=o)
    # weighted sums in place, inside the rows
    route = dip.ExpertRoute(4, 3, 2, "cuda")
    dip.dip_route_experts(ctx, torch.randn((4, 3), generator=g, device="cuda"), route)
    out = torch.randn((8, 256), generator=g, device="cuda")
    before = out.clone()
    for first in (0, 3):
        refused(dip.dip_combine_rows, out, route, out.view(torch.bfloat16).view(16, 256)[first:first + 4])
    work = dip.ExpertWork(4, 2, w, "cuda")
    x = torch.randn((4, 256), generator=g, device="cuda").bfloat16()
    refused(dip.dip_expert_mlp, w, x, work, work.out.view(torch.bfloat16).view(16, 256)[4:8], route=route)
    torch.cuda.synchronize()
    assert torch.equal(rows.scales, scales) and torch.equal(out, before) and (h.values.view(torch.uint8) == 3).all()


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("top_k", [0, 2])
def test_the_block_in_place(ctx, wtype, top_k):
    """y over x: x is used up when y is written."""
    g = gen_of(2)
    w = block(g, wtype == "fp8", 5 if top_k else 1, 288, 416)
    x = torch.randn((70, 288), generator=g, device="cuda").bfloat16()
    work, y, route = dip.ExpertWork(70, top_k, w, "cuda"), torch.zeros_like(x), None
    if top_k:
        route = dip.ExpertRoute(70, 5, top_k, "cuda")
        dip.dip_route_experts(ctx, torch.randn((70, 5), generator=g, device="cuda"), route)
    dip.dip_expert_mlp(ctx, w, x, work, y, route=route)
    dip.dip_expert_mlp(ctx, w, x, work, x, route=route)
    assert torch.equal(x, y)


@pytest.mark.parametrize("rows", [1, 7, 40])
def test_rows_and_scales_that_the_launch_in_front_writes(ctx, rows):
    """A product starts before the launch that stages its rows is through: new rows and scales in the same buffers, launch after
    launch, give what they give one at a time."""
    g = gen_of(4)
    m = dip.GroupedMatrix(*eu.matrix(g, True, 1, 608, 1280))
    x = [(torch.randn((rows, 1280), generator=g, device="cuda") * 4.0 ** (i % 7 - 3)).bfloat16() for i in range(40)]
    staged, want = dip.Rows(rows, 1280, dip.W_FP8_B128, "cuda"), []
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


# ---- waits that run out ------------------------------------------------------------------------------------------------
def test_a_grouped_product_that_gives_up_waits_for_its_copies_and_a_reset_mends_the_context():
    """Warps that wait in vain end the others' waits, and no block leaves while what it has asked for is under way (alone, and in
    pairs of which either block is ahead).  Then cut tiles, whose parts meet, on the same context."""
    c = dip.Context(0)
    try:
        report = torch.full((dip.SELFTEST_GROUP_CASES, 2), -1, dtype=torch.int64, device="cuda")
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        c.selftest_group_waits(2000, report)
        b.record()
        assert c.device_status() == dip.DEVICE_WAIT_TIMEOUT
        # twice the limit each, and not the second that the other waits have
        assert 2 * 2 * dip.SELFTEST_GROUP_CASES <= a.elapsed_time(b) < 500
        # copies under way: of the last five steps, those that each block has asked for
        under_way = [3, 5, 4 + 4, 5 + 5, 5 + 1, 5 + 2, 1 + 5, 2 + 4]
        assert report.tolist() == [[n, n] for n in under_way]
        c.reset_device_status()
        g = gen_of(3)
        for fp8 in (False, True):
            for counts in ([1, 0, 3], [70, 0, 90], [400, 0, 250]):
                w, x = eu.matrix(g, fp8, 3, 352, 8192), eu.rows_of(g, fp8, sum(counts), 8192)
                o = eu.offsets(counts)
                y = torch.zeros((sum(counts), 352), device="cuda")
                dip.dip_grouped_product(c, dip.GroupedMatrix(*w), dip.Rows.of(*x), y, offset=o)
                want, bound = eu.product64(*w, eu.values64(*x), o)
                eu.assert_within(y, want, eu.rounded(want, bound, torch.float32), "y")
        assert c.device_status() == dip.DEVICE_OK
        for limit, bad in ((0, report), (2_000_000, report), (1000, report[:3]), (1000, report.int()), (1000, report.cpu())):
            with pytest.raises(dip.DipError):
                c.selftest_group_waits(limit, bad)
    finally:
        torch.cuda.synchronize()
        c.close()


# ---- sizes at the ends of what a call takes ----------------------------------------------------------------------------
@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d_in,d_out", [(32768, 32), (32, 32768)])
@pytest.mark.parametrize("rows", [1, 40])
def test_widest_and_narrowest(ctx, wtype, d_in, d_out, rows):
    g, fp8 = gen_of(d_in + rows), wtype == "fp8"
    w, x = eu.matrix(g, fp8, 1, d_out, d_in), eu.rows_of(g, fp8, rows, d_in)
    y = torch.zeros((rows, d_out), device="cuda")
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), dip.Rows.of(*x), y)
    want, bound = eu.product64(*w, eu.values64(*x))
    eu.assert_within(y, want, eu.rounded(want, bound, torch.float32), "y")


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
def test_most_experts(ctx, wtype):
    """512 experts, 16 for each token; a group of many rows, and most of few or none."""
    g, fp8 = gen_of(6), wtype == "fp8"
    w = block(g, fp8, 512, 64, 96)
    z = torch.randn((50, 512), generator=g, device="cuda")
    z[:, 511] = 9
    x = torch.randn((50, 64), generator=g, device="cuda").bfloat16()
    route, work, y = dip.ExpertRoute(50, 512, 16, "cuda"), dip.ExpertWork(50, 16, w, "cuda"), torch.zeros_like(x)
    dip.dip_route_experts(ctx, z, route)
    dip.dip_expert_mlp(ctx, w, x, work, y, route=route)
    assert int(route.offset[-1] - route.offset[-2]) == 50
    want, bound = eu.product64(w.down.values, w.down.scales, eu.values64(work.h.values, work.h.scales), route.offset)
    eu.assert_within(work.out, want, bound, "out")
    at, share = route.token_row.long(), route.weight.double()[:, :, None]
    total, off = (want[at] * share).sum(1), ((bound[at] + want[at].abs() * 2.0 ** -23 * 17) * share).sum(1)
    eu.assert_within(y, total, eu.rounded(total, off, torch.bfloat16), "y")


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("top_k", [1, 3])
def test_a_batch_of_nothing_but_padding(ctx, wtype, top_k):
    g = gen_of(7)
    w = block(g, wtype == "fp8", 4, 160, 288)
    x = torch.full((33, 160), float("nan"), device="cuda", dtype=torch.bfloat16)
    route, work, y = dip.ExpertRoute(33, 4, top_k, "cuda"), dip.ExpertWork(33, top_k, w, "cuda"), torch.full_like(x, 5.0)
    for t in (work.rows.values, work.h.values):
        t.view(torch.uint8).fill_(0x7f)                            # (NaN codes; finite bfloat16)
    work.out.fill_(float("nan"))
    dip.dip_route_experts(ctx, torch.full((33, 4), -float("inf"), device="cuda"), route)
    dip.dip_expert_mlp(ctx, w, x, work, y, route=route)
    assert (y == 0).all() and torch.isnan(work.out).all()


@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
def test_positions_beyond_32_bits(ctx, wtype):
    """Rows and outputs of more than 2^31 values (and 2^32 bytes): the last rows' values, and the rows in front of them."""
    tokens, top_k, d_in, d_out = 65536, 16, 2080, 4128
    rows_there = tokens * top_k
    g, fp8 = gen_of(8), wtype == "fp8"
    z = torch.zeros((tokens, 16), device="cuda")                   # every token, every expert: rows of a group are the tokens
    x = torch.randn((tokens, d_in), generator=g, device="cuda").bfloat16()
    w = eu.matrix(g, fp8, 16, d_out, d_in)
    route, staged = dip.ExpertRoute(tokens, 16, top_k, "cuda"), dip.Rows(rows_there, d_in, WTYPES[wtype], "cuda")
    dip.dip_route_experts(ctx, z, route)
    dip.dip_stage_rows(ctx, x, staged, route=route)
    y = torch.empty((rows_there, d_out), device="cuda", dtype=torch.bfloat16)
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), staged, y, offset=route.offset)
    for e in (0, 7, 8, 15):
        some = torch.tensor([0, 1, 127, 128, 40000, tokens - 1], device="cuda")
        r = some + e * tokens
        want_rows = x[some]
        if fp8:
            want_rows, s = eu.quantise(want_rows)
            assert torch.equal(staged.scales[r], s)
        assert torch.equal(staged.values[r].view(torch.uint8), want_rows.view(torch.uint8))
        want, bound = eu.product64(w[0][e:e + 1], None if w[1] is None else w[1][e:e + 1], eu.values64(want_rows, s if fp8 else None))
        eu.assert_within(y[r], want, eu.rounded(want, bound, torch.bfloat16), "y of expert %d" % e)
    del staged
    out = torch.zeros((rows_there, d_in), device="cuda")           # 8.7 GB
    out[-tokens:] = x.float()
    got = torch.empty_like(x)
    dip.dip_combine_rows(ctx, out, route, got)
    # only the last expert's rows are not zero; its share of 16 equal logits
    want = x.double() * route.weight[:, -1:].double()
    eu.assert_within(got, want, eu.rounded(want, want.abs() * 2.0 ** -24, torch.bfloat16), "weighted sum")


# ---- graphs ------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("wtype", ["bf16", "fp8"])
@pytest.mark.parametrize("tokens", [1, 300, 4500])
def test_the_first_call_of_a_context_may_be_a_captured_one(wtype, tokens):
    """Nothing has to have run before (kernels of few, some and many rows for each expert)."""
    g = gen_of(9)
    c = dip.Context(0)
    try:
        w = block(g, wtype == "fp8", 4, 160, 288)
        x, z = torch.randn((tokens, 160), generator=g, device="cuda").bfloat16(), torch.randn((tokens, 4), generator=g, device="cuda")
        route, work, y = dip.ExpertRoute(tokens, 4, 2, "cuda"), dip.ExpertWork(tokens, 2, w, "cuda"), torch.zeros_like(x)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dip.dip_route_experts(c, z, route)
            dip.dip_expert_mlp(c, w, x, work, y, route=route)
        graph.replay()
        got = y.clone()
        dip.dip_route_experts(c, z, route)
        dip.dip_expert_mlp(c, w, x, work, y, route=route)
        assert torch.equal(got, y) and y.float().abs().max() > 0
        assert c.device_status() == dip.DEVICE_OK
        del graph
    finally:
        torch.cuda.synchronize()
        c.close()
