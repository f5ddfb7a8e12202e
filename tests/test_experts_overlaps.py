"""Buffers of a router's, a grouped product's or an expert block's call that share memory: what a launch writes must not overlap
what it reads or what else it writes.  The library's own argument checks, compiled for the host alone with launchers that only
count (no GPU needed; the addresses are never followed)."""
import ctypes as C
import os
import subprocess

import pytest

pytest.importorskip("torch")
import paper_2412_01380_b200 as dip

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TOKENS, EXPERTS, TOP_K, D, F = 5, 4, 2, 160, 96
ROWS, BASE, APART = TOKENS * TOP_K, 1 << 40, 1 << 20
BF16, FP8 = dip.W_BF16, dip.W_FP8_B128

STUB = """
#include "common.cuh"
static int launches;
static dip_ctx context;
extern "C" cudaError_t cudaGetDevice(int *device) { *device = 0; return cudaSuccess; }
extern "C" dip_ctx *stub_context() { return &context; }
extern "C" int stub_launches() { const int n = launches; launches = 0; return n; }
dip_status dip_launch_route(dip_ctx *, const void *, bool, bool, const dip_expert_route &, cudaStream_t) { ++launches; return DIP_OK; }
dip_status dip_launch_stage_rows(dip_ctx *, const void *, int, int, const dip_expert_route *, bool, void *, float *, cudaStream_t)
{ ++launches; return DIP_OK; }
dip_status dip_launch_combine_rows(dip_ctx *, const float *, const dip_expert_route &, int, void *, cudaStream_t) { ++launches; return DIP_OK; }
dip_status dip_launch_grouped(dip_ctx *, const dip_grouped_matrix &, const dip_grouped_matrix *, const void *, const float *, int,
                              const int32_t *, void *, bool, float *, cudaStream_t) { ++launches; return DIP_OK; }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    folder = tmp_path_factory.mktemp("experts")
    (folder / "stub.cc").write_text(STUB)
    out = str(folder / "libexperts.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-x", "c++", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(dip._HERE, "csrc"), "-I", os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"),
                    os.path.join(dip._HERE, "csrc", "experts.cu"), str(folder / "stub.cc"), "-o", out], check=True)
    lib = C.CDLL(out)
    lib.stub_context.restype = C.c_void_p
    return lib


def blocks(d):
    return -(-d // 128)


def matrix(wtype, experts, d_out, d_in, at, name):
    return dip.GroupedMatrixStruct(wtype, experts, d_out, d_in, at[name], at.get(name + "_scales"))


def weights(wtype, experts, d_out, d_in, name):
    sizes = {name: experts * d_out * d_in * (2 if wtype == BF16 else 1)}
    if wtype == FP8:
        sizes[name + "_scales"] = experts * blocks(d_out) * blocks(d_in) * 4
    return sizes


def rows(wtype, n, d, name):
    sizes = {name: n * d * (2 if wtype == BF16 else 1)}
    if wtype == FP8:
        sizes[name + "_scales"] = n * blocks(d) * 4
    return sizes


ROUTE = {"expert": ROWS * 4, "weight": ROWS * 4, "offset": (EXPERTS + 1) * 4, "row_token": ROWS * 4, "token_row": ROWS * 4}
X, Y = {"x": TOKENS * D * 2}, {"y": TOKENS * D * 2}


def route_struct(at):
    return dip.ExpertRouteStruct(TOKENS, EXPERTS, TOP_K, 0, *(at[n] for n in ROUTE))


def route_call(bf16):
    sizes = dict(ROUTE, logits=TOKENS * EXPERTS * (2 if bf16 else 4))
    return sizes, set(ROUTE), lambda lib, c, at: lib.dip_route_experts(c, C.c_void_p(at["logits"]), bf16, 1, C.byref(route_struct(at)), None)


def stage_call(wtype, routed):
    out = rows(wtype, ROWS if routed else TOKENS, D, "rows")
    sizes = dict(X, **out)
    if routed:
        sizes.update(ROUTE)

    def call(lib, c, at):
        return lib.dip_stage_rows(c, C.c_void_p(at["x"]), TOKENS, D, C.byref(route_struct(at)) if routed else None, wtype,
                                  C.c_void_p(at["rows"]), C.c_void_p(at.get("rows_scales")), None)
    # (a route's experts and weights are no business of this launch, but no buffer that it may lose either)
    return sizes, set(out), call


def product_call(wtype, f32):
    sizes = dict(weights(wtype, EXPERTS, F, D, "w"), offset=ROUTE["offset"], y=ROWS * F * (4 if f32 else 2), **rows(wtype, ROWS, D, "rows"))

    def call(lib, c, at):
        return lib.dip_grouped_product(c, C.byref(matrix(wtype, EXPERTS, F, D, at, "w")), C.c_void_p(at["rows"]),
                                       C.c_void_p(at.get("rows_scales")), ROWS, C.c_void_p(at["offset"]), C.c_void_p(at["y"]), f32, None)
    return sizes, {"y"}, call


def gate_up_call(wtype):
    out = rows(wtype, ROWS, F, "h")
    sizes = dict(weights(wtype, EXPERTS, F, D, "gate"), **weights(wtype, EXPERTS, F, D, "up"), **rows(wtype, ROWS, D, "rows"), **out,
                 offset=ROUTE["offset"])

    def call(lib, c, at):
        return lib.dip_grouped_gate_up(c, C.byref(matrix(wtype, EXPERTS, F, D, at, "gate")), C.byref(matrix(wtype, EXPERTS, F, D, at, "up")),
                                       C.c_void_p(at["rows"]), C.c_void_p(at.get("rows_scales")), ROWS, C.c_void_p(at["offset"]),
                                       C.c_void_p(at["h"]), C.c_void_p(at.get("h_scales")), None)
    return sizes, set(out), call


def combine_call():
    sizes = dict(ROUTE, out=ROWS * D * 4, **Y)
    return sizes, {"y"}, lambda lib, c, at: lib.dip_combine_rows(c, C.c_void_p(at["out"]), C.byref(route_struct(at)), D, C.c_void_p(at["y"]), None)


def mlp_call(wtype, routed):
    experts, n = (EXPERTS, ROWS) if routed else (1, TOKENS)
    staged = routed or wtype == FP8
    sizes = dict(X, **Y, **weights(wtype, experts, F, D, "gate"), **weights(wtype, experts, F, D, "up"), **weights(wtype, experts, D, F, "down"),
                 **rows(wtype, n, F, "h"))
    if staged:
        sizes.update(rows(wtype, n, D, "rows"))
    if routed:
        sizes.update(ROUTE, out=n * D * 4)

    def call(lib, c, at):
        work = dip.ExpertWorkStruct(at.get("rows"), at.get("rows_scales"), at["h"], at.get("h_scales"), at.get("out"))
        return lib.dip_expert_mlp(c, C.byref(matrix(wtype, experts, F, D, at, "gate")), C.byref(matrix(wtype, experts, F, D, at, "up")),
                                  C.byref(matrix(wtype, experts, D, F, at, "down")), C.c_void_p(at["x"]), TOKENS,
                                  C.byref(route_struct(at)) if routed else None, C.byref(work), C.c_void_p(at["y"]), None)
    return sizes, {"rows", "rows_scales", "h", "h_scales", "out", "y"} & set(sizes), call


def used_up(name, other, sizes):
    """dip_expert_mlp: the launch that writes `name` comes behind the last one that reads or writes `other`."""
    last = {"x": 1 if "rows" in sizes else 2, "rows": 2, "rows_scales": 2, "h": 3, "h_scales": 3, "out": 4}
    first = {"rows": 1, "rows_scales": 1, "h": 2, "h_scales": 2, "out": 3, "y": 4 if "out" in sizes else 3}
    return name in first and other in last and first[name] > last[other]


CALLS = {"route_f32": route_call(0), "route_bf16": route_call(1), "combine": combine_call()}
CALLS.update({"stage_%d_%d" % (w, r): stage_call(w, r) for w in (BF16, FP8) for r in (False, True)})
CALLS.update({"product_%d_%d" % (w, f): product_call(w, f) for w in (BF16, FP8) for f in (0, 1)})
CALLS.update({"gate_up_%d" % w: gate_up_call(w) for w in (BF16, FP8)})
CALLS.update({"mlp_%d_%d" % (w, r): mlp_call(w, r) for w in (BF16, FP8) for r in (False, True)})


@pytest.mark.parametrize("name", list(CALLS))
def test_what_a_launch_writes_overlaps_nothing(lib, name):
    sizes, written, call = CALLS[name]
    apart = {n: BASE + i * APART for i, n in enumerate(sizes)}
    context = C.c_void_p(lib.stub_context())

    def outcome(**moved):
        status = call(lib, context, dict(apart, **moved))
        return status, lib.stub_launches()

    status, launches = outcome()
    assert status == dip.OK and launches >= 1
    for w in sorted(written):
        for other in sizes:
            if other == w:
                continue
            at = apart[other]
            # neighbours
            for here in ((at + sizes[other] + 15) // 16 * 16, at - (sizes[w] + 15) // 16 * 16):
                assert outcome(**{w: here}) == (dip.OK, launches), (w, other)
            # the same place; its last bytes; its first bytes
            for here in (at, at + (sizes[other] - 1) // 16 * 16, at - (sizes[w] - 1) // 16 * 16):
                free = name.startswith("mlp") and (used_up(w, other, sizes) or used_up(other, w, sizes))
                want = (dip.OK, launches) if free else (dip.ERR_INVALID_ARG, 0)
                assert outcome(**{w: here}) == want, (w, other)
