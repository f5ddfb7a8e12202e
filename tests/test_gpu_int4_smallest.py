"""Products with 4-bit weights at the smallest numbers that rows and scales can hold."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2412_01380_b200 as dip
import int4_util as iu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = dip.Context(0)
    yield c
    assert c.device_status() == dip.DEVICE_OK
    c.close()


# Scales, and the powers of two between which the lowest bit of x is then: (code - 8) * scale * x has 22 bits at most, none of them below 2^-149,
# so binary32 holds it and no order of exact steps loses anything.
RANGES = {"large scales": ([2.0 ** 10, 1027.0, -65504.0, 2.0 ** 15], -133, -100),
          "one": ([1.0, -1.0, 2.0, 0.5], -133, -100),
          "small scales": ([2.0 ** -24, -(2.0 ** -24), 3 * 2.0 ** -24, 2.0 ** -20], -125, -100)}


@pytest.mark.parametrize("kind", list(RANGES))
@pytest.mark.parametrize("d_out", [64, 65536])                     # (the second one: with 256 rows by the kernel for many rows)
@pytest.mark.parametrize("rows", [1, 9, 256])
def test_every_code_with_the_smallest_inputs(ctx, rows, d_out, kind):
    """One input at a time: y is (code - 8) * scale * x exactly, down to the smallest bfloat16 number."""
    some, lowest, highest = RANGES[kind]
    g = torch.Generator(device="cuda")
    g.manual_seed(rows)
    d_in = 256
    codes = torch.randint(0, 256, (1, d_out, d_in // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.tensor(some, device="cuda").half()[torch.randint(0, 4, (1, 2, d_out), generator=g, device="cuda")]
    # 1 .. 255 times a power of two: eight bits, of which the lowest may be a subnormal number's
    x = torch.randint(1, 256, (d_in,), generator=g, device="cuda").double()
    x = torch.diag(x * torch.exp2(torch.randint(lowest, highest, (d_in,), generator=g, device="cuda").double()))
    first = {1: 77, 9: 128, 256: 0}[rows]
    x[first, first] = 255 * 2.0 ** lowest
    if rows > 1:
        x[first + 1, first + 1] = 2.0 ** lowest
    bf = x.bfloat16()
    assert torch.equal(bf.double(), x)
    part = bf[first:first + rows].contiguous()
    y = torch.full((rows, d_out), math.nan, device="cuda")
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(codes, scales), dip.Rows.of(part), y)
    want = part.double() @ iu.weights64(codes, scales, 0).t()
    assert torch.equal(want.float().double(), want)
    assert torch.equal(y.double(), want)
