"""Products with 4-bit weights by each of their two kernels, at every size: the rule that chooses between them moves no case away from a test.

The tests of test_gpu_int4.py run here again, on a context that takes one kernel for all calls."""
import math
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

import paper_2412_01380_b200 as dip
import expert_util as eu
import int4_util as iu
import test_gpu_int4 as t
from test_gpu_int4 import (  # noqa: F401
    test_a_prompt_and_then_decode_steps_from_the_same_arrays, test_a_scale_that_is_not_finite_stays_in_its_output,
    test_a_value_that_is_not_finite_stays_in_its_row, test_dense_block_and_in_place, test_dense_gate_up, test_dense_product,
    test_every_code_and_scale, test_gate_up_groups, test_gate_up_loads, test_gate_up_sizes, test_large_and_small_inputs, test_mixture,
    test_more_tiles_than_fit_at_once, test_offsets_are_cut_off, test_product_groups, test_product_loads, test_product_sizes,
    test_rows_that_the_launch_in_front_writes, test_same_bits_again_on_another_stream_and_from_a_graph, test_the_most_experts_and_rows,
    test_the_widest, test_two_graphs_of_one_context)
from test_gpu_int4_smallest import test_every_code_with_the_smallest_inputs  # noqa: F401

pytestmark = pytest.mark.gpu
KERNELS = {"few": 1, "many": 2}


def context(kernel):
    return dip.Context(0, int4_kernel=KERNELS[kernel])


@pytest.fixture(scope="module", params=list(KERNELS))
def ctx(request):
    c = context(request.param)
    yield c
    assert c.device_status() == dip.DEVICE_OK
    c.close()


@pytest.fixture(scope="module")
def kernels():
    """One context for each kernel, and one that chooses."""
    made = {name: context(name) for name in KERNELS}
    made["chosen"] = dip.Context(0)
    yield made
    for c in made.values():
        assert c.device_status() == dip.DEVICE_OK
        c.close()


def sums(c, m, rows):
    y = torch.zeros((rows.n_rows, m.d_out), device="cuda")
    dip.dip_grouped_product(c, m, rows, y)
    return y


@pytest.mark.parametrize("rows,d_in,d_out,which", [
    (1, 5120, 17920, "few"), (8, 4096, 102400, "few"), (16, 256, 192, "few"), (77, 2080, 1056, "few"),
    (200, 5120, 17920, "many"), (2048, 4096, 4096, "many"), (4000, 1280, 4160, "many"), (256, 256, 65536, "many")])
def test_which_kernel_a_call_takes(kernels, rows, d_in, d_out, which):
    """The order of additions tells them apart: of thousands of sums by both, some differ in their last bit."""
    g = t.gen_of(rows)
    m, x = dip.GroupedMatrix(*iu.matrix(g, 1, d_out, d_in)), dip.Rows.of(t.rows_of(g, rows, d_in))
    y = {name: sums(c, m, x) for name, c in kernels.items()}
    assert not torch.equal(y["few"], y["many"])
    assert torch.equal(y["chosen"], y[which])


@pytest.mark.parametrize("counts", [[1], [3, 0, 17], [31, 33, 0, 65], [128, 1, 260, 7]])
@pytest.mark.parametrize("d_in,d_out", [(32, 64), (64, 160), (96, 416), (160, 96), (192, 544), (224, 32), (1216, 288), (4128, 160), (4192, 288)])
def test_inputs_that_end_inside_a_group(ctx, d_in, d_out, counts):
    """32, 64 and 96 inputs of the last group, alone and behind others, in tiles that are whole and that are cut."""
    t.check_product(ctx, counts, d_in, d_out, torch.float32, extra=1, seed=d_in)
    t.check_gate_up(ctx, counts, d_in, d_out, seed=d_in)


@pytest.mark.parametrize("neighbour", [math.nan, math.inf])
@pytest.mark.parametrize("counts", [[5, 5, 5], [33, 31, 100], [130, 126, 20]])
def test_rows_of_other_experts(ctx, counts, neighbour):
    """A piece of rows that is copied holds the next expert's rows, too: what these are changes nothing."""
    g, n = t.gen_of(21), sum(counts)
    w, x, offset = iu.matrix(g, 3, 288, 352), t.rows_of(g, n, 352), eu.offsets(counts)
    y = [torch.zeros((n, 288), device="cuda") for _ in range(2)]
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), dip.Rows.of(x), y[0], offset=offset)
    a, b = counts[0], counts[0] + counts[1]
    x[a:b] = neighbour
    dip.dip_grouped_product(ctx, dip.GroupedMatrix(*w), dip.Rows.of(x), y[1], offset=offset)
    assert torch.equal(y[0][:a], y[1][:a]) and torch.equal(y[0][b:], y[1][b:])
    assert not torch.isfinite(y[1][a:b]).any()


@pytest.mark.parametrize("rows", [3, 40, 300])
@pytest.mark.parametrize("kernel", list(KERNELS))
def test_two_contexts_at_once_and_types_in_turn(kernel, rows):
    """Each context has its own workspace: products whose tiles are cut, side by side on two streams, in turn with bfloat16 ones that
    use the same workspace."""
    g = t.gen_of(14)
    m = [dip.GroupedMatrix(*iu.matrix(g, 1, 416, 8192)), dip.GroupedMatrix(eu.matrix(g, False, 1, 416, 8192)[0])]
    x = [dip.Rows.of(t.rows_of(g, rows, 8192)) for _ in range(2)]
    contexts = [context(kernel), context(kernel)]
    alone = [sums(contexts[0], w, r) for r in x for w in m]
    torch.cuda.synchronize()
    streams, both = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(y) for y in alone]
    for _ in range(20):
        for i, (s, c) in enumerate(zip(streams, contexts)):
            with torch.cuda.stream(s):
                for j, w in enumerate(m):
                    dip.dip_grouped_product(c, w, x[i], both[2 * i + j])
    torch.cuda.synchronize()
    for c in contexts:
        assert c.device_status() == dip.DEVICE_OK
        c.close()
    for a, b in zip(alone, both):
        assert torch.equal(a, b)


@pytest.mark.parametrize("tokens", [5, 150])
def test_a_block_whose_kernels_take_turns(kernels, tokens):
    """Contexts of either kernel give the same block but for the order of additions in it."""
    g = t.gen_of(tokens)
    gate, up, down, w = t.weights(g, 1, 544, 800)
    x = t.rows_of(g, tokens, 544)
    work, h = dip.ExpertWork(tokens, 0, w, "cuda"), iu.gated64(gate, up, x)
    want, mass = h[0] @ iu.weights64(*down, 0).t(), h[0].abs() @ iu.weights64(*down, 0).abs().t()
    # the sums of h and of y, half a step of h and half a step of y
    off = h[1] @ iu.weights64(*down, 0).abs().t() + mass * (800 + 2 * 7) * 2.0 ** -23 + mass * 2.0 ** -8 + want.abs() * 2.0 ** -8
    for name in ("few", "many", "chosen", "many", "few"):
        y = torch.full((tokens, 544), math.nan, device="cuda", dtype=torch.bfloat16)
        dip.dip_expert_mlp(kernels[name], w, x, work, y)
        eu.assert_within(y, want, off, name)


FIRST_CALL_UNDER_CAPTURE = """
import sys, torch
sys.path[:0] = [%r, %r]
import paper_2412_01380_b200 as dip, int4_util as iu
g = torch.Generator(device="cuda")
ctx = dip.Context(0, int4_kernel=%d)
m = [dip.GroupedMatrix(*iu.matrix(g, 1, 416, 1280)) for _ in range(2)]
rows = [dip.Rows.of(torch.randn((n, 1280), generator=g, device="cuda").bfloat16()) for n in (3, 12, 300)]
ys = [torch.zeros((r.n_rows, 416), device="cuda") for r in rows]
hs = [dip.Rows(r.n_rows, 416, dip.W_BF16, "cuda") for r in rows]
for h in hs:
    h.values.zero_()

def calls():
    for r, y, h in zip(rows, ys, hs):
        dip.dip_grouped_product(ctx, m[0], r, y)
        dip.dip_grouped_gate_up(ctx, m[0], m[1], r, h)

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    calls()
assert not any(y.any() for y in ys) and not any(h.values.any() for h in hs)
graph.replay()
torch.cuda.synchronize()
got = [y.clone() for y in ys] + [h.values.clone() for h in hs]
calls()
assert all(torch.equal(a, b) for a, b in zip(got, ys + [h.values for h in hs])) and all(v.any() for v in got)
assert ctx.device_status() == dip.DEVICE_OK
print("as told")
"""


@pytest.mark.parametrize("kernel", list(KERNELS))
def test_first_call_under_capture(kernel):
    """A process whose very first call is a captured one of this kernel."""
    here = os.path.dirname(os.path.abspath(__file__))
    code = FIRST_CALL_UNDER_CAPTURE % (os.path.dirname(here), here, KERNELS[kernel])
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "as told" in out.stdout, out.stderr[-2000:]


def test_the_choice_of_a_kernel_is_one_of_three():
    for wrong in (-1, 3):
        with pytest.raises(dip.DipError) as e:
            dip.Context(0, int4_kernel=wrong)
        assert e.value.status == dip.ERR_INVALID_ARG
