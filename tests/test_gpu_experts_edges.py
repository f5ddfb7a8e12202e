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
