"""The choice of tokens from logits against its definition in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2412_01380_b200 as dip
import int4_util as iu
import sample_util as su

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


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


def column(values, n, dtype=F32):
    """Each of the values in turn, one a row."""
    return None if values is None else torch.tensor([values[i % len(values)] for i in range(n)], device="cuda", dtype=dtype)


def check(ctx, z, u, temperature=None, top_k=None, top_p=None, min_p=None):
    """A call and each row's reference.  A probability has one rounding to binary32, and the whole is a sum of weights that are each off by
    2^-46 of the largest: 2^-28 for 2^18 of them."""
    n = z.shape[0]
    how = dict(temperature=column(temperature, n), top_k=column(top_k, n, torch.int32), top_p=column(top_p, n), min_p=column(min_p, n))
    token = torch.full((n + 2,), -77, device="cuda", dtype=torch.int32)
    prob = torch.full((n + 2,), -77.0, device="cuda")
    dip.dip_sample_tokens(ctx, z, u, token[:n], prob=prob[:n], **how)
    assert (token[n:] == -77).all() and (prob[n:] == -77).all()
    again = torch.full((n,), -77, device="cuda", dtype=torch.int32)
    dip.dip_sample_tokens(ctx, z, u, again, **how)                 # without prob
    assert torch.equal(again, token[:n])
    got_t, got_p, rows, us = token[:n].tolist(), prob[:n].tolist(), z.cpu(), u.tolist()
    settings = {k: v.tolist() for k, v in how.items() if v is not None}
    for r in range(n):
        t, p, edge = su.choose(rows[r], us[r], **{k: v[r] for k, v in settings.items()})
        assert got_t[r] == t, (r, got_t[r], t, edge, {k: v[r] for k, v in settings.items()})
        assert abs(got_p[r] - p) <= p * (2.0 ** -24 + 2.0 ** -27), (r, got_p[r], p)
    return got_t


def logits(g, n, vocab, dtype, spread=2.0):
    z = torch.randn((n, vocab), generator=g, device="cuda") * spread
    z[:, :: max(1, vocab // 7)] += 5.0
    return z.to(dtype)


MODES = {
    "plain": dict(temperature=[0.7, 1.0, 1.3, 0.05, 20.0]),
    "none": dict(),
    "greedy": dict(temperature=[0.0, -1.0, math.nan]),
    "top_k": dict(top_k=[1, 2, 40, 500, 5000, 0, -3]),
    "top_p": dict(top_p=[0.9, 0.5, 0.99, 0.1, 1.0, 0.999, 0.0], temperature=[0.8, 1.0, 1.7]),
    "min_p": dict(min_p=[0.05, 0.5, 1.0, 0.001, 0.0, 2.0]),
    "all": dict(temperature=[0.8, 1.2, 0.0, 1.0], top_k=[50, 1000, 3, 0, 7], top_p=[0.9, 0.6, 1.0], min_p=[0.0, 0.02]),
}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("n,vocab", [(9, 1), (9, 2), (5, 33), (33, 1000), (7, 4097), (5, 32064), (3, 50257)])
def test_modes(ctx, n, vocab, mode, dtype):
    g = gen_of(vocab)
    check(ctx, logits(g, n, vocab, dtype), torch.rand((n,), generator=g, device="cuda"), **MODES[mode])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,vocab", [(1, 262144), (2, 151001), (3, 262143), (75, 20011), (160, 9000), (300, 1500)])
def test_every_share_of_a_row(ctx, n, vocab, dtype):
    """One block per row to eight, whole and ragged parts, blocks without a logit."""
    g = gen_of(n)
    z = logits(g, n, vocab, dtype)
    for mode in ("all", "top_p"):
        check(ctx, z, torch.rand((n,), generator=g, device="cuda"), **MODES[mode])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mode", ["plain", "top_p", "all", "min_p"])
def test_rows_that_do_not_stay_in_shared_memory(ctx, mode, dtype):
    """More rows than blocks find room for, and longer ones than fit beside what else a block has: they are read again."""
    g = gen_of(11)
    z = logits(g, 310, 36011, dtype)
    z[5], z[6, 100:] = -math.inf, -math.inf
    check(ctx, z[:, 3:], torch.rand((310,), generator=g, device="cuda"), **MODES[mode])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_closed_logits(ctx, dtype):
    g = gen_of(1)
    z = logits(g, 24, 5003, dtype)
    closed = torch.rand(z.shape, generator=g, device="cuda") < 0.6
    z[:8].masked_fill_(closed[:8], -math.inf)
    z[8:16].masked_fill_(closed[8:16], torch.finfo(dtype).min)     # the type's lowest value is open, far below
    z[16:20].masked_fill_(closed[16:20], math.nan)
    z[3], z[11], z[17] = -math.inf, torch.finfo(dtype).min, math.nan
    z[5], z[5, 4321] = -math.inf, -30.0                            # one is left
    z[20, [7, 9, 4000]] = math.inf
    z[21] = math.inf
    z[22, 100] = torch.finfo(dtype).max
    got = []
    for mode in MODES:
        got.append(check(ctx, z, torch.rand((24,), generator=g, device="cuda"), **MODES[mode]))
    for t in got:
        assert t[3] == -1 and t[17] == -1 and t[11] >= 0 and t[5] == 4321 and t[20] in (7, 9, 4000) and t[22] == 100


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [700, 30011, 120001])
def test_ties(ctx, vocab, dtype):
    """The lower index is in front: among all that are equal, among a few values, and 0 beside -0."""
    g = gen_of(2)
    z = torch.zeros((12, vocab), device="cuda")
    z[1] = -3.25
    z[2:5] = torch.randint(0, 3, (3, vocab), generator=g, device="cuda").float()
    z[5:8] = torch.randint(-20, 1, (3, vocab), generator=g, device="cuda") * 0.125
    z[8:10] = torch.where(torch.rand((2, vocab), generator=g, device="cuda") < 0.5, 0.0, -0.0)
    z[10:] = (torch.randn((2, vocab), generator=g, device="cuda") * 4).round() / 4
    u = torch.rand((12,), generator=g, device="cuda")
    for how in (dict(top_k=[1, vocab // 3, vocab // 2, 600]), dict(top_p=[0.3, 0.7, 0.9]), dict(top_k=[vocab // 2], top_p=[0.51, 0.2], temperature=[0.9]),
                dict(), dict(temperature=[0.0]), dict(top_p=[0.25], min_p=[0.5])):
        check(ctx, z.to(dtype), u, **how)
    # all alike: index u * n
    t = torch.empty((12,), device="cuda", dtype=torch.int32)
    dip.dip_sample_tokens(ctx, z.to(dtype)[:1], u[:1], t[:1])
    assert abs(int(t[0]) - int(float(u[0]) * vocab)) <= 1


def test_logits_that_crowd(ctx):
    """Most of a row in one bin of any even division: far below one logit, within a hair of one another, over all magnitudes."""
    g = gen_of(3)
    vocab = 40009
    z = torch.randn((8, vocab), generator=g, device="cuda")
    z[0] *= 1e-3
    z[0, 17] = 60.0
    z[1] = 5.0 + z[1] * 1e-6
    z[2] = torch.exp(z[2] * 20)                                    # 10^-37 .. 10^37
    z[3] = -torch.exp(z[3] * 15)
    z[4] = z[4] * 1e-38                                            # some of them subnormal
    z[5, :30000] = -1e30
    z[6] = 1e6 + z[6]
    z[7, ::2] = -200.0
    u = torch.rand((8,), generator=g, device="cuda")
    for how in (dict(top_k=[3, 3000, 20000]), dict(top_k=[25000, 39000]), dict(top_p=[0.5, 0.9], temperature=[1.0, 30.0, 1e-3, 1e6]), dict(),
                dict(temperature=[1e30, math.inf, 1e-30, 1e-42]), dict(top_k=[30001, 12000], top_p=[0.9], temperature=[100.0])):
        check(ctx, z, u, **how)


def test_the_ends_of_the_settings(ctx):
    g = gen_of(4)
    z = logits(g, 40, 999, F32)
    u = torch.rand((40,), generator=g, device="cuda")
    u[:9] = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 5.0, -1.0, math.nan, math.inf, 2.0 ** -149, 0.5], device="cuda")
    for how in (dict(), dict(top_p=[1.0 - 2.0 ** -24, 2.0 ** -100, -1.0, math.nan, 3.0]), dict(top_k=[999, 998, 1000, 2 ** 31 - 1, -2 ** 31]),
                dict(min_p=[math.nan, -1.0, 1.0, math.inf, 2.0 ** -120])):
        check(ctx, z, u, **how)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [600, 5003])
@pytest.mark.parametrize("kind", ["alike", "huge", "tiny"])
def test_temperatures_and_logits_at_the_ends_of_their_range(ctx, kind, vocab, dtype):
    """An infinite temperature (all alike, with any min_p), differences of logits that pass the largest binary32 number, and temperatures and
    differences below the smallest normal one."""
    g = gen_of(vocab)
    n = 12
    z = torch.randn((n, vocab), generator=g, device="cuda")
    temperature = [math.inf]
    if kind == "huge":
        z, temperature = (z * 1.5e38).clamp(-3.3e38, 3.3e38), [math.inf, 1e38, 2.5e38, 3e37]
    if kind == "tiny":
        step = 2.0 ** -133                      # bfloat16's smallest number
        z, temperature = torch.randint(-40, 40, (n, vocab), generator=g, device="cuda").double() * step, [4 * step, 2.0 ** -130, 2.0 ** -126]
    z = z.to(dtype)
    z[:, 5] = -math.inf
    u = torch.rand((n,), generator=g, device="cuda")
    check(ctx, z, u, temperature=temperature)
    check(ctx, z, u, temperature=temperature, min_p=[1.0, 0.5, 3.0, 0.03])
    check(ctx, z, u, temperature=temperature, top_p=[0.5, 0.9])
    check(ctx, z, u, temperature=temperature, top_k=[7, 300], min_p=[0.2, 1.0, 0.0])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_anywhere(ctx, dtype):
    """Rows that are apart, and that start anywhere."""
    g = gen_of(5)
    whole = logits(g, 11, 3007, dtype)
    u = torch.rand((11,), generator=g, device="cuda")
    for view in (whole[:, :3000], whole[:, 1:2999], whole[:, 5:], whole[1:, 3:2500], whole[::2, 7:1000], whole[3:4, 1:]):
        n = view.shape[0]
        check(ctx, view, u[:n].clone(), **MODES["all"])


def test_shares_follow_the_probabilities(ctx):
    """65536 evenly spaced numbers through one row: each token gets its share to within one number at either end of its range."""
    g = gen_of(6)
    z = (torch.randn((1, 97), generator=g, device="cuda") * 2).expand(65536, 97).contiguous()
    u = torch.arange(65536, device="cuda") / 65536.0
    token = torch.empty((65536,), device="cuda", dtype=torch.int32)
    dip.dip_sample_tokens(ctx, z, u, token)
    share = torch.bincount(token.long(), minlength=97)
    want = torch.softmax(z[0].double(), 0) * 65536
    assert ((share - want).abs() <= 1.0).all() and (token[1:] >= token[:-1]).all()


# ---- streams, graphs, repetition ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("n,vocab", [(1, 32064), (70, 20011)])
def test_again_on_another_stream_and_from_a_graph(ctx, n, vocab):
    g = gen_of(7)
    z, u = logits(g, n, vocab, BF16), torch.rand((n,), generator=g, device="cuda")
    how = dict(temperature=column([0.9], n), top_k=column([50, 0], n, torch.int32), top_p=column([0.9], n))
    token, prob = torch.zeros((n,), device="cuda", dtype=torch.int32), torch.zeros((n,), device="cuda")

    def call():
        dip.dip_sample_tokens(ctx, z, u, token, prob=prob, **how)

    call()
    first = token.clone(), prob.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            token.zero_()
            call()
            assert torch.equal(token, first[0]) and torch.equal(prob, first[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    u.copy_(torch.rand((n,), generator=g, device="cuda"))
    z.copy_(logits(g, n, vocab, BF16))
    graph.replay()
    replayed = token.clone()
    token.zero_()
    call()
    assert torch.equal(token, replayed)
    check(ctx, z, u, temperature=[0.9], top_k=[50, 0], top_p=[0.9])


def test_calls_at_once(ctx):
    """No workspace is shared, so one context serves several streams."""
    g = gen_of(8)
    z = [logits(g, 5, 50000 + 13 * i, F32) for i in range(4)]
    u = torch.rand((5,), generator=g, device="cuda")
    p = column([0.9], 5)
    want = []
    for v in z:
        t = torch.zeros((5,), device="cuda", dtype=torch.int32)
        dip.dip_sample_tokens(ctx, v, u, t, top_p=p)
        want.append(t)
    got = [torch.zeros_like(t) for t in want]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in z]
    for _ in range(10):
        for s, v, t in zip(streams, z, got):
            with torch.cuda.stream(s):
                dip.dip_sample_tokens(ctx, v, u, t, top_p=p)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


FIRST_CALLS_UNDER_CAPTURE = """
import sys, torch
sys.path[:0] = [%r, %r]
import paper_2412_01380_b200 as dip, int4_util as iu
g = torch.Generator(device="cuda")
ctx = dip.Context(0)
m = dip.GroupedMatrix(*iu.matrix(g, 1, 416, 1280))
rows = [dip.Rows.of(torch.randn((n, 1280), generator=g, device="cuda").bfloat16()) for n in (3, 12, 2000)]
ys = [torch.zeros((r.n_rows, 416), device="cuda") for r in rows]
z, u = torch.randn((5, 9000), generator=g, device="cuda"), torch.rand((5,), generator=g, device="cuda")
token = torch.full((5,), -7, device="cuda", dtype=torch.int32)
k = torch.full((5,), 40, device="cuda", dtype=torch.int32)

def calls():
    for r, y in zip(rows, ys):
        dip.dip_grouped_product(ctx, m, r, y)
    dip.dip_sample_tokens(ctx, z, u, token, top_k=k)

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
assert (token == -7).all() and not any(y.any() for y in ys)
graph.replay()
torch.cuda.synchronize()
got = [y.clone() for y in ys] + [token.clone()]
calls()
assert all(torch.equal(a, b) for a, b in zip(got, ys + [token])) and all(y.any() for y in ys) and (token >= 0).all()
assert ctx.device_status() == dip.DEVICE_OK
print("as told")
"""


def test_first_calls_under_capture():
    """A process whose very first calls are captured."""
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    out = subprocess.run([sys.executable, "-c", FIRST_CALLS_UNDER_CAPTURE % (os.path.dirname(here), here)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "as told" in out.stdout, out.stderr[-2000:]


@pytest.mark.parametrize("n", [1, 3, 40])
def test_a_step_of_a_decode_loop(ctx, n):
    """A block with 4-bit weights, the 4-bit head's logits (a vocabulary beyond the widest input) and the token drawn from them, launch after
    launch without a wait, and the same replayed from a graph."""
    g = gen_of(9)
    d, f, vocab = 512, 1408, 40992
    w = dip.ExpertWeights(*(dip.GroupedMatrix(*iu.matrix(g, 1, a, b)) for a, b in ((f, d), (f, d), (d, f))))
    codes, scales = iu.matrix(g, 1, vocab, d)
    head = dip.GroupedMatrix(codes, (scales.float() * 2.0 ** -3).half())
    x, h = torch.randn((n, d), generator=g, device="cuda").bfloat16(), torch.zeros((n, d), device="cuda", dtype=BF16)
    work, z = dip.ExpertWork(n, 0, w, "cuda"), torch.zeros((n, vocab), device="cuda")
    rows, u = dip.Rows.of(h), torch.rand((n,), generator=g, device="cuda")
    t, k, p = column([400.0], n), column([300], n, torch.int32), column([0.9], n)
    token = torch.zeros((n,), device="cuda", dtype=torch.int32)

    def step():
        dip.dip_expert_mlp(ctx, w, x, work, h)
        dip.dip_grouped_product(ctx, head, rows, z)
        dip.dip_sample_tokens(ctx, z, u, token, temperature=t, top_k=k, top_p=p)

    step()
    want, bound = iu.product64(head.values, head.scales, h)
    assert ((z.double() - want).abs() <= bound).all()
    for r in range(n):
        assert int(token[r]) == su.choose(z[r].cpu(), float(u[r]), 400.0, 300, 0.9)[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x.copy_(torch.randn((n, d), generator=g, device="cuda"))
    graph.replay()
    replayed = token.clone()
    step()
    assert torch.equal(token, replayed)


# ---- refusals that need a device ---------------------------------------------------------------------------------------
def test_refused_calls_launch_nothing(ctx):
    z, u = torch.zeros((4, 100), device="cuda"), torch.zeros((4,), device="cuda")
    token = torch.full((4,), 9, device="cuda", dtype=torch.int32)

    def refused(*args, **kw):
        with pytest.raises(dip.DipError) as e:
            dip.dip_sample_tokens(ctx, *args, **kw)
        assert e.value.status == dip.ERR_INVALID_ARG

    for bad in (z.half(), z.double(), z.cpu(), z[0], z.t(), z[:, ::2], z[:0], torch.zeros((4, 262145), device="cuda"), z[:1].expand(4, 100)):
        refused(bad, u, token)
    refused(z, u[:3], token)
    refused(z, u.double(), token)
    refused(z, None, token)
    refused(z, u, None)
    refused(z, u, token.long())
    refused(z, u, token, prob=u[:3])
    refused(z, u, token, prob=u)                                   # over what is read
    refused(z, u, token, prob=token.view(F32))                     # over what is written
    refused(z, u, z.view(torch.int32)[1, :4])
    refused(z, u, token, top_k=u)
    refused(z, u, token, temperature=u.cpu())
    refused(z, u, token, top_p=torch.zeros((8,), device="cuda")[::2])
    torch.cuda.synchronize()
    assert (token == 9).all()
