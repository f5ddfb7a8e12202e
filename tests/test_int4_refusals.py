"""What the library refuses of products with 4-bit weights, on the host alone (no GPU needed): a fake context's device is never the
current one, so what is checked here is that the calls return, and what the binding says before them."""
import ctypes as C
import types

import pytest

torch = pytest.importorskip("torch")
import paper_2412_01380_b200 as dip

CTX = types.SimpleNamespace(device=0, handle=None)
INT4 = dip.W_INT4_G128


def test_the_binding_refuses_matrices_of_the_wrong_kind():
    codes, scales = torch.zeros((2, 64, 48), dtype=torch.uint8), torch.zeros((2, 1, 64), dtype=torch.float16)
    for values, s in ((codes, scales), (codes, None), (codes[0], scales[0]), (codes, scales.float()), (codes.to(torch.int8), scales)):
        with pytest.raises(dip.DipError):                          # (none is on a device)
            dip.GroupedMatrix(values, s)


def test_rows_of_4_bit_weights_are_bfloat16():
    with pytest.raises(dip.DipError):
        dip.Rows(4, 64, INT4, "cpu")
    w = types.SimpleNamespace(wtype=INT4, d_model=64, d_ff=96)
    work = dip.ExpertWork(4, 2, w, "cpu")
    assert work.wtype == INT4 and work.rows.wtype == work.h.wtype == dip.W_BF16 and work.rows.scales is None and work.h.scales is None
    assert dip.ExpertWork(4, 0, w, "cpu").rows is None


@pytest.mark.parametrize("pair", [(dip.W_BF16, INT4), (INT4, dip.W_BF16), (INT4, dip.W_FP8_B128)])
def test_gate_and_up_are_of_one_type(pair):
    gate, up = (types.SimpleNamespace(device=0, wtype=t, d_in=64, d_out=96, n_experts=1, ref=None) for t in pair)
    rows, h = dip.Rows(4, 64, dip.W_BF16, "cpu"), dip.Rows(4, 96, dip.W_BF16, "cpu")
    rows.device = h.device = 0
    rows.n_rows = 4
    with pytest.raises(dip.DipError):
        dip.dip_grouped_gate_up(CTX, gate, up, rows, h)


def test_null_arguments_of_the_library():
    lib = C.CDLL(dip.LIB_PATH)
    m = dip.GroupedMatrixStruct(INT4, 1, 64, 96, None, None)
    assert lib.dip_grouped_product(None, C.byref(m), None, None, 1, None, None, 0, None) == dip.ERR_INVALID_ARG
    assert lib.dip_grouped_gate_up(None, C.byref(m), C.byref(m), None, None, 1, None, None, None, None) == dip.ERR_INVALID_ARG


# ---- buffers that share memory: the library's own checks, compiled for the host with launchers that only count -------------------------
ROWS, EXPERTS, D, F, BASE, APART = 10, 4, 160, 96, 1 << 40, 1 << 20


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    import os
    import subprocess

    from test_experts_overlaps import ROOT, STUB
    folder = tmp_path_factory.mktemp("int4")
    (folder / "stub.cc").write_text(STUB)
    out = str(folder / "libexperts.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-x", "c++", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(dip._HERE, "csrc"), "-I", os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include"),
                    os.path.join(dip._HERE, "csrc", "experts.cu"), str(folder / "stub.cc"), "-o", out], check=True)
    lib = C.CDLL(out)
    lib.stub_context.restype = C.c_void_p
    return lib


SIZES = {"w": EXPERTS * F * D // 2, "w_scales": EXPERTS * 2 * F * 2, "rows": ROWS * D * 2, "offset": (EXPERTS + 1) * 4, "y": ROWS * F * 4}


def product(lib, at, d_out=F, d_in=D, up=False):
    c = C.c_void_p(lib.stub_context())
    m = dip.GroupedMatrixStruct(INT4, EXPERTS, d_out, d_in, at["w"], at["w_scales"])
    o, y, x = C.c_void_p(at["offset"]), C.c_void_p(at["y"]), C.c_void_p(at["rows"])
    if up:
        return lib.dip_grouped_gate_up(c, C.byref(m), C.byref(m), x, None, ROWS, o, y, None, None)
    return lib.dip_grouped_product(c, C.byref(m), x, None, ROWS, o, y, 1, None)


@pytest.mark.parametrize("read", ["w", "w_scales", "rows", "offset"])
def test_a_product_does_not_write_what_it_reads(lib, read):
    at = {name: BASE + i * APART for i, name in enumerate(SIZES)}
    assert product(lib, at) == dip.OK and lib.stub_launches() == 1
    for first, refused in ((at[read] + SIZES[read] - 16, True), (at[read] + -(-SIZES[read] // 16) * 16, False),
                           (at[read] - SIZES["y"] + 16, True), (at[read] - SIZES["y"], False)):
        status = product(lib, dict(at, y=first))
        assert (status, lib.stub_launches()) == ((dip.ERR_INVALID_ARG, 0) if refused else (dip.OK, 1)), (read, first)


@pytest.mark.parametrize("d_out,d_in,up,ok", [
    (262144, 160, False, True), (262176, 160, False, False), (32800, 160, False, True), (32800, 160, True, False), (32768, 160, True, True),
    (96, 32768, False, True), (96, 32800, False, False), (96, 144, False, False), (80, 160, False, False), (0, 160, False, False)])
def test_widths(lib, d_out, d_in, up, ok):
    at = {name: BASE + i * (1 << 36) for i, name in enumerate(SIZES)}
    assert product(lib, at, d_out, d_in, up) == (dip.OK if ok else dip.ERR_INVALID_ARG)
    assert lib.stub_launches() == int(ok)


@pytest.mark.parametrize("name", ["w", "w_scales", "rows", "offset", "y"])
def test_addresses_are_whole_pieces_of_16_bytes(lib, name):
    at = {n: BASE + i * APART for i, n in enumerate(SIZES)}
    assert product(lib, dict(at, **{name: at[name] + 8})) == dip.ERR_INVALID_ARG
    if name != "offset":                                           # (none: one expert)
        assert product(lib, dict(at, **{name: None})) == dip.ERR_INVALID_ARG
    assert lib.stub_launches() == 0
