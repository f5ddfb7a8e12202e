"""4-bit products and the choice of tokens whose weights, outputs or logits lie beyond what 32 bits count."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2412_01380_b200 as dip
import expert_util as eu
import int4_util as iu
import sample_util as su
from test_gpu_int4 import gen_of, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=[1, 2])
def ctx(request):
    c = dip.Context(0, int4_kernel=request.param)
    yield c
    assert c.device_status() == dip.DEVICE_OK
    c.close()


def test_outputs(ctx):
    """9000 rows of the widest head, binary32: 2^31 outputs and more."""
    g, n, d_in, d_out = gen_of(1), 9000, 32, 262144
    w, x = iu.matrix(g, 1, d_out, d_in), rows_of(g, n, d_in)
    y = torch.full((n + 1, d_out), math.nan, device="cuda")
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), dip.Rows.of(x), y)
    assert torch.isnan(y[n]).all()
    for a in (0, 4090, 8185, 8900):                                # 2^30 outputs are 4096 rows
        want, bound = iu.product64(*w, x[a:a + 100])
        eu.assert_within(y[a:a + 100], want, eu.rounded(want, bound, torch.float32), "y")


@pytest.mark.parametrize("gated", [False, True])
def test_weights(ctx, gated):
    """40 experts of 8192 to 32768: 5.4 GB of codes, with rows for the first one, one in the middle and the last ones."""
    g, experts, d_in, d_out = gen_of(2), 40, 8192, 32768
    counts = [0] * experts
    counts[0], counts[17], counts[38], counts[39] = 3, 1, 20, 6
    ws = [iu.matrix(g, experts, d_out, d_in) for _ in range(2 if gated else 1)]
    n, offset = sum(counts), eu.offsets(counts)
    x = rows_of(g, n, d_in)
    if gated:
        x = (x.float() * 2.0 ** -6).bfloat16()                     # (sums of gate and up of a few units)
        h = dip.Rows(n, d_out, dip.W_BF16, "cuda")
        dip.dip_grouped_gate_up(ctx, *(dip.GroupedMatrix(*w) for w in ws), dip.Rows.of(x), h, offset=offset)
        y, of = h.values, lambda *a: iu.gated64(*a)
    else:
        y, of = torch.zeros((n, d_out), device="cuda", dtype=torch.bfloat16), lambda *a: iu.product64(*a[0], a[1])
        dip.dip_grouped_product(ctx, dip.GroupedMatrix(*ws[0]), dip.Rows.of(x), y, offset=offset)
    for e, a, b in eu.groups(offset, n, experts):
        if b > a:
            want, bound = of(*((c[e:e + 1], s[e:e + 1]) for c, s in ws), x[a:b])
            eu.assert_within(y[a:b], want, eu.rounded(want, bound, torch.bfloat16), "expert %d" % e)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_logits(ctx, dtype):
    """Rows of the largest vocabulary, 2^31 items and more behind the first one, by their number and by their distance."""
    g, vocab = gen_of(3), 262144
    z = torch.empty((8200, vocab), device="cuda", dtype=dtype)
    z.normal_(generator=g)
    u = torch.rand((8200,), generator=g, device="cuda")
    p, k = torch.full((8200,), 0.9, device="cuda"), torch.full((8200,), 50, device="cuda", dtype=torch.int32)
    for rows, numbers in ((z, u), (z[::4099], u[:3].clone())):
        n = rows.shape[0]
        token = torch.full((n,), -7, device="cuda", dtype=torch.int32)
        dip.dip_sample_tokens(ctx, rows, numbers, token, top_k=k[:n], top_p=p[:n])
        for r in {0, 1, n // 2, n - 2, n - 1}:
            assert int(token[r]) == su.choose(rows[r].cpu(), float(numbers[r]), top_k=50, top_p=float(p[0]))[0]
