"""Thin Python binding of the sm_100a DIP / DIP-CA sparse decode-MLP library (include/dip.h).

Argument marshalling only: every step of the method runs in the CUDA kernels of
`libdip.so`.  PyTorch supplies device memory and streams.  There is no CPU
fallback: importing this package without the built library raises ImportError.

Functions carry the names of the C entry points they call.
"""
import ctypes as C
import os
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdip.so")

W_F32, W_BF16, W_INT4_G128, W_FP8_B128 = 0, 1, 2, 3
MAX_D, MAX_BATCH, INT4_GROUP, CACHE_META_INTS = 32768, 16, 128, 8
FP8_BLOCK, MAX_EXPERTS, MAX_TOP_K, MAX_TOKENS = 128, 512, 16, 65536
SELFTEST_GROUP_CASES = 8
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_CUDA, ERR_WORKSPACE = 0, 1, 2, 3, 4
DEVICE_OK, DEVICE_WAIT_TIMEOUT, DEVICE_TIER_INCONSISTENT = 0, 1, 2

if not os.path.exists(LIB_PATH):
    raise ImportError(
        "%s is missing: build it with `python paper_2412_01380_b200/build.py` "
        "(nvcc, sm_100a).  This package has no fallback path." % LIB_PATH)
_lib = C.CDLL(LIB_PATH)

_vp, _i32, _f32 = C.c_void_p, C.c_int, C.c_float


class MlpWeightsStruct(C.Structure):
    _fields_ = [("wtype", C.c_int32), ("d_model", C.c_int32), ("d_ff", C.c_int32), ("reserved", C.c_int32),
                ("gate_up", _vp), ("gate_up_scales", _vp), ("down", _vp), ("down_scales", _vp)]


class CacheStateStruct(C.Structure):
    _fields_ = [("d", C.c_int32), ("capacity", C.c_int32), ("stamp", _vp), ("meta", _vp), ("count", _vp),
                ("policy", C.c_int32), ("reserved", C.c_int32)]


class StepOutputsStruct(C.Structure):
    _fields_ = [("mask_x", _vp), ("idx_x", _vp), ("h", _vp), ("mask_h", _vp), ("idx_h", _vp),
                ("union_counts", _vp)]


class OptionsStruct(C.Structure):
    _fields_ = [("max_d", C.c_int32), ("max_batch", C.c_int32), ("gemv_segment_bytes", C.c_int32),
                ("gemv_copy_ring", C.c_int32), ("coarse_min_d", C.c_int32), ("wait_limit_us", C.c_int32),
                ("select_in_product", C.c_int32), ("reserved", C.c_int32 * 3)]


class StackProbeStruct(C.Structure):
    _fields_ = [("x", _vp), ("mask_x", _vp), ("h", _vp), ("mask_h", _vp), ("y", _vp)]


_lib.dip_create.restype = _i32
_lib.dip_create.argtypes = [C.POINTER(_vp), _i32]
_lib.dip_create_ex.restype = _i32
_lib.dip_create_ex.argtypes = [C.POINTER(_vp), _i32, C.POINTER(OptionsStruct)]
_lib.dip_reset_device_status.restype = _i32
_lib.dip_reset_device_status.argtypes = [_vp, _vp]
_lib.dip_selftest_bounded_wait.restype = _i32
_lib.dip_selftest_bounded_wait.argtypes = [_vp, _i32, _vp, _vp]
_lib.dip_selftest_group_waits.restype = _i32
_lib.dip_selftest_group_waits.argtypes = [_vp, _i32, _vp, _vp]
_lib.dip_selftest_block_waits.restype = _i32
_lib.dip_selftest_block_waits.argtypes = [_vp, _i32, C.POINTER(CacheStateStruct), _vp, _vp]
_lib.dip_destroy.restype = _i32
_lib.dip_destroy.argtypes = [_vp]
_lib.dip_status_string.restype = C.c_char_p
_lib.dip_status_string.argtypes = [_i32]
_lib.dip_last_error.restype = C.c_char_p
_lib.dip_last_error.argtypes = [_vp]
_lib.dip_sm_count.restype = _i32
_lib.dip_sm_count.argtypes = [_vp]
_lib.dip_device_status.restype = _i32
_lib.dip_device_status.argtypes = [_vp, C.POINTER(C.c_int), _vp]
_lib.dip_packed_bytes.restype = C.c_size_t
_lib.dip_packed_bytes.argtypes = [_i32, _i32, _i32, _i32]
_lib.dip_pack_weights.restype = _i32
_lib.dip_pack_weights.argtypes = [_vp, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _vp,
                                  C.POINTER(MlpWeightsStruct), _vp]
_lib.dip_mask_topk.restype = _i32
_lib.dip_mask_topk.argtypes = [_vp, _vp, _i32, _i32, _i32, _vp, _vp, _vp]
_lib.dip_ca_mask.restype = _i32
_lib.dip_ca_mask.argtypes = [_vp, _vp, _i32, _i32, _f32, C.POINTER(CacheStateStruct), _vp, _vp, _vp]
for _name in ("dip_sparse_gemv_gate_up", "dip_sparse_gemv_down"):
    getattr(_lib, _name).restype = _i32
    getattr(_lib, _name).argtypes = [_vp, C.POINTER(MlpWeightsStruct), _vp, _i32, _vp, _i32, _vp, _vp, _vp]
_lib.dip_select_gemv_gate_up.restype = _i32
_lib.dip_select_gemv_gate_up.argtypes = [_vp, C.POINTER(MlpWeightsStruct), _vp, _i32, _f32, C.POINTER(CacheStateStruct),
                                         C.POINTER(CacheStateStruct), _vp, _vp, _vp]
_lib.dip_select_gemv_down.restype = _i32
_lib.dip_select_gemv_down.argtypes = [_vp, C.POINTER(MlpWeightsStruct), _vp, _i32, _f32, C.POINTER(CacheStateStruct),
                                      _vp, _vp, _vp]
_lib.dip_mlp_step.restype = _i32
_lib.dip_mlp_step.argtypes = [_vp, C.POINTER(MlpWeightsStruct), _vp, _i32, _i32, _i32, _f32,
                              C.POINTER(CacheStateStruct), C.POINTER(CacheStateStruct), _vp,
                              C.POINTER(StepOutputsStruct), _vp]
_lib.dip_residual_rmsnorm.restype = _i32
_lib.dip_residual_rmsnorm.argtypes = [_vp, _vp, _vp, _i32, _i32, _vp, _vp]
_lib.dip_stack_step.restype = _i32
_lib.dip_stack_step.argtypes = [_vp, _i32, C.POINTER(MlpWeightsStruct), _vp, _i32, _i32, _i32, _f32,
                                C.POINTER(CacheStateStruct), C.POINTER(CacheStateStruct), _vp, _vp, _vp]
_lib.dip_stack_step_probed.restype = _i32
_lib.dip_stack_step_probed.argtypes = [_vp, _i32, C.POINTER(MlpWeightsStruct), _vp, _i32, _i32, _i32, _f32,
                                       C.POINTER(CacheStateStruct), C.POINTER(CacheStateStruct), _vp,
                                       C.POINTER(StackProbeStruct), _vp]


class TierStruct(C.Structure):
    _fields_ = [("d", C.c_int32), ("capacity", C.c_int32), ("staging", C.c_int32), ("reserved", C.c_int32),
                ("row_bytes", C.c_uint64), ("backing", _vp), ("arena", _vp), ("slot", _vp), ("loc", _vp),
                ("fetch", _vp), ("split", _vp), ("counters", _vp)]


_lib.dip_mlp_step_tiered.restype = _i32
_lib.dip_mlp_step_tiered.argtypes = [_vp, C.POINTER(MlpWeightsStruct), C.POINTER(TierStruct), C.POINTER(TierStruct),
                                     _vp, _i32, _i32, _f32, C.POINTER(CacheStateStruct),
                                     C.POINTER(CacheStateStruct), _vp, C.POINTER(StepOutputsStruct), _vp]


class NeuronWeightsStruct(C.Structure):
    _fields_ = [("wtype", C.c_int32), ("d_model", C.c_int32), ("d_ff", C.c_int32), ("reserved", C.c_int32),
                ("gate", _vp), ("up", _vp), ("down", _vp)]


PRUNE_BY_GATE, PRUNE_BY_UP = 0, 1
_lib.dip_mlp_step_neuron_pruned.restype = _i32
_lib.dip_mlp_step_neuron_pruned.argtypes = [_vp, C.POINTER(NeuronWeightsStruct), _i32, _vp, _i32, _vp,
                                            _vp, _vp, _vp, _vp, _vp]
_lib.dip_sparse_gemv_down_noalloc.restype = _i32
_lib.dip_sparse_gemv_down_noalloc.argtypes = [C.POINTER(MlpWeightsStruct), _vp, _vp, _i32, _vp, _vp]



class GroupedMatrixStruct(C.Structure):
    _fields_ = [("wtype", C.c_int32), ("n_experts", C.c_int32), ("d_out", C.c_int32), ("d_in", C.c_int32),
                ("values", _vp), ("scales", _vp)]


class ExpertRouteStruct(C.Structure):
    _fields_ = [("n_tokens", C.c_int32), ("n_experts", C.c_int32), ("top_k", C.c_int32), ("reserved", C.c_int32),
                ("expert", _vp), ("weight", _vp), ("offset", _vp), ("row_token", _vp), ("token_row", _vp)]


class ExpertWorkStruct(C.Structure):
    _fields_ = [("rows", _vp), ("row_scales", _vp), ("h", _vp), ("h_scales", _vp), ("out", _vp)]


_lib.dip_route_experts.restype = _i32
_lib.dip_route_experts.argtypes = [_vp, _vp, _i32, _i32, C.POINTER(ExpertRouteStruct), _vp]
_lib.dip_stage_rows.restype = _i32
_lib.dip_stage_rows.argtypes = [_vp, _vp, _i32, _i32, C.POINTER(ExpertRouteStruct), _i32, _vp, _vp, _vp]
_lib.dip_grouped_product.restype = _i32
_lib.dip_grouped_product.argtypes = [_vp, C.POINTER(GroupedMatrixStruct), _vp, _vp, _i32, _vp, _vp, _i32, _vp]
_lib.dip_grouped_gate_up.restype = _i32
_lib.dip_grouped_gate_up.argtypes = [_vp, C.POINTER(GroupedMatrixStruct), C.POINTER(GroupedMatrixStruct), _vp, _vp, _i32,
                                     _vp, _vp, _vp, _vp]
_lib.dip_combine_rows.restype = _i32
_lib.dip_combine_rows.argtypes = [_vp, _vp, C.POINTER(ExpertRouteStruct), _i32, _vp, _vp]
_lib.dip_expert_mlp.restype = _i32
_lib.dip_expert_mlp.argtypes = [_vp, C.POINTER(GroupedMatrixStruct), C.POINTER(GroupedMatrixStruct),
                                C.POINTER(GroupedMatrixStruct), _vp, _i32, C.POINTER(ExpertRouteStruct),
                                C.POINTER(ExpertWorkStruct), _vp, _vp]

EXPORTED = ["dip_create", "dip_create_ex", "dip_destroy", "dip_status_string", "dip_last_error", "dip_sm_count",
            "dip_device_status", "dip_reset_device_status", "dip_selftest_bounded_wait", "dip_selftest_block_waits", "dip_selftest_group_waits", "dip_stack_step_probed",
            "dip_trace_begin", "dip_trace_reset", "dip_trace_read", "dip_trace_end",
            "dip_packed_bytes", "dip_pack_weights", "dip_mask_topk", "dip_ca_mask",
            "dip_sparse_gemv_gate_up", "dip_sparse_gemv_down", "dip_select_gemv_gate_up", "dip_select_gemv_down",
            "dip_mlp_step",
            "dip_residual_rmsnorm", "dip_stack_step", "dip_mlp_step_tiered", "dip_mlp_step_neuron_pruned",
            "dip_sparse_gemv_down_noalloc",
            "dip_route_experts", "dip_stage_rows", "dip_grouped_product", "dip_grouped_gate_up", "dip_combine_rows",
            "dip_expert_mlp"]


class TraceRecord(C.Structure):
    _fields_ = [("kind", C.c_int32), ("reserved", C.c_int32), ("t_start_ns", C.c_uint64),
                ("t_ready_ns", C.c_uint64), ("t_end_ns", C.c_uint64), ("t_aux_ns", C.c_uint64)]


TRACE_KINDS = {1: "select", 2: "select_ca", 3: "cache_update", 4: "gemv_gate_up", 5: "gemv_down",
               6: "tier_books", 7: "tier_fetch", 9: "rowdot", 10: "grouped_gate_up", 11: "grouped_product"}
for _name in ("dip_trace_begin", "dip_trace_reset", "dip_trace_end"):
    getattr(_lib, _name).restype = _i32
    getattr(_lib, _name).argtypes = [_vp]
_lib.dip_trace_read.restype = _i32
_lib.dip_trace_read.argtypes = [_vp, C.POINTER(TraceRecord), _i32, C.POINTER(C.c_int)]


class DipError(RuntimeError):
    def __init__(self, status: int, detail: str = ""):
        self.status = status
        msg = _lib.dip_status_string(status).decode()
        super().__init__("%s (status %d)%s" % (msg, status, (": " + detail) if detail else ""))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _current_stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _raw_stream() -> int:
    # the current device's current stream without a Stream object around it: 0.2 us instead of 3.2 of the 13 us that the host
    # spends on one step of two launches (seen in a step's time only where the host is the bound)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


# (both names are torch's own; builds of torch without CUDA lack them)
_stream = _raw_stream if hasattr(torch._C, "_cuda_getCurrentRawStream") and hasattr(torch._C, "_cuda_getDevice") else _current_stream


class Context:
    """A dip_ctx: scratch workspace on one device.  Not for concurrent use from several streams."""

    def __init__(self, device: int = 0, max_d: int = 0, max_batch: int = 0, gemv_segment_bytes: int = 0,
                 gemv_copy_ring: bool = False, coarse_min_d: int = 0, wait_limit_us: int = 0,
                 select_in_product: int = 0):
        """The keyword arguments are the fields of dip_options (0 = the library's default)."""
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2412_01380_b200 needs a CUDA device; there is no CPU path")
        h = _vp()
        opt = OptionsStruct(int(max_d), int(max_batch), int(gemv_segment_bytes), int(bool(gemv_copy_ring)),
                            int(coarse_min_d), int(wait_limit_us), int(select_in_product))
        st = _lib.dip_create_ex(C.byref(h), int(device), C.byref(opt))
        if st != OK:
            raise DipError(st, "dip_create_ex")
        self.handle = h
        self.device = int(device)

    def check(self, st: int) -> None:
        if st != OK:
            raise DipError(st, _lib.dip_last_error(self.handle).decode())

    @property
    def sm_count(self) -> int:
        return _lib.dip_sm_count(self.handle)

    def device_status(self) -> int:
        """Waits for the current stream; 0 unless a kernel gave up a bounded wait."""
        out = C.c_int(-1)
        self.check(_lib.dip_device_status(self.handle, C.byref(out), _stream()))
        return out.value

    def reset_device_status(self) -> None:
        self.check(_lib.dip_reset_device_status(self.handle, _stream()))

    def selftest_bounded_wait(self, limit_us: int, waited_ns: Optional[torch.Tensor] = None) -> None:
        """Enqueue the tiny kernel whose bounded wait runs out (device status becomes 1)."""
        self.check(_lib.dip_selftest_bounded_wait(self.handle, int(limit_us), _ptr(waited_ns), _stream()))

    def selftest_group_waits(self, limit_us: int, report: torch.Tensor) -> None:
        """report: contiguous int64 [SELFTEST_GROUP_CASES, 2] on the context's device."""
        if (report.dtype is not torch.int64 or report.get_device() != self.device or not report.is_contiguous() or
                report.shape != (SELFTEST_GROUP_CASES, 2)):
            raise DipError(ERR_INVALID_ARG, "report must be contiguous int64 [%d, 2] on the context's device" % SELFTEST_GROUP_CASES)
        self.check(_lib.dip_selftest_group_waits(self.handle, int(limit_us), _ptr(report), _stream()))

    def selftest_block_waits(self, limit_us: int, st: "CacheState", mask_bits: torch.Tensor) -> None:
        """Enqueue the kernel whose waits between thread blocks run out (device status becomes 1, st stays as it is)."""
        self.check(_lib.dip_selftest_block_waits(self.handle, int(limit_us), C.byref(st.struct), _ptr(mask_bits), _stream()))

    def trace_begin(self) -> None:
        self.check(_lib.dip_trace_begin(self.handle))

    def trace_reset(self) -> None:
        self.check(_lib.dip_trace_reset(self.handle))

    def trace_end(self) -> None:
        self.check(_lib.dip_trace_end(self.handle))

    def trace_read(self):
        """Records of the launches that ran since the last reset: list of dicts with times in
        microseconds relative to the earliest start."""
        buf = (TraceRecord * 1024)()
        n = C.c_int(0)
        self.check(_lib.dip_trace_read(self.handle, buf, 1024, C.byref(n)))
        recs = [buf[i] for i in range(n.value)]
        if not recs:
            return []
        t0 = min(r.t_start_ns for r in recs)
        return [{"kind": TRACE_KINDS.get(r.kind, str(r.kind)), "start": (r.t_start_ns - t0) / 1e3,
                 "ready": (r.t_ready_ns - t0) / 1e3, "end": (r.t_end_ns - t0) / 1e3,
                 "aux": (r.t_aux_ns - t0) / 1e3 if r.t_aux_ns else None} for r in recs]

    def close(self) -> None:
        if self.handle:
            _lib.dip_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class MlpWeights:
    """Packed weights of one MLP block (device tensors owned here) plus the C struct naming them."""

    def __init__(self, wtype: int, d_model: int, d_ff: int, device):
        self.wtype, self.d_model, self.d_ff = int(wtype), int(d_model), int(d_ff)
        sizes = [_lib.dip_packed_bytes(wtype, d_model, d_ff, w) for w in range(4)]
        if sizes[0] == 0:
            raise DipError(ERR_INVALID_ARG, "unsupported weight type or shape")
        self.gate_up = torch.empty(sizes[0], dtype=torch.uint8, device=device)
        self.down = torch.empty(sizes[1], dtype=torch.uint8, device=device)
        self.gate_up_scales = torch.empty(sizes[2], dtype=torch.uint8, device=device) if sizes[2] else None
        self.down_scales = torch.empty(sizes[3], dtype=torch.uint8, device=device) if sizes[3] else None
        self.struct = MlpWeightsStruct(self.wtype, self.d_model, self.d_ff, 0, _ptr(self.gate_up),
                                       _ptr(self.gate_up_scales), _ptr(self.down), _ptr(self.down_scales))

    @property
    def nbytes(self) -> int:
        return sum(t.numel() for t in (self.gate_up, self.down, self.gate_up_scales, self.down_scales)
                   if t is not None)


class CacheState:
    """Column-cache state of one masked layer input: stamp int32[d], meta int32[8] on the device."""

    def __init__(self, d: int, capacity: int, device, policy: str = "lru"):
        assert policy in ("lru", "lfu")
        self.d, self.capacity, self.policy = int(d), int(capacity), policy
        self.stamp = torch.full((d,), -1, dtype=torch.int32, device=device)
        self.meta = torch.zeros(CACHE_META_INTS, dtype=torch.int32, device=device)
        self.count = torch.zeros(d, dtype=torch.int32, device=device) if policy == "lfu" else None
        self.struct = CacheStateStruct(self.d, self.capacity, _ptr(self.stamp), _ptr(self.meta), _ptr(self.count),
                                       1 if policy == "lfu" else 0, 0)

    def load(self, stamp, n_resident: int, step: int, counters=(0, 0, 0, 0)) -> None:
        self.stamp.copy_(torch.as_tensor(stamp, dtype=torch.int32))
        self.meta.copy_(torch.tensor([n_resident, step, *counters, 0, 0], dtype=torch.int32))


def dip_packed_bytes(wtype: int, d_model: int, d_ff: int, which: int) -> int:
    return int(_lib.dip_packed_bytes(wtype, d_model, d_ff, which))


def dip_pack_weights(ctx: Context, wtype: int, d_model: int, d_ff: int,
                     Wg: torch.Tensor, Wu: torch.Tensor, Wd: torch.Tensor,
                     Sg: Optional[torch.Tensor] = None, Su: Optional[torch.Tensor] = None,
                     Sd: Optional[torch.Tensor] = None, out: Optional[MlpWeights] = None) -> MlpWeights:
    """Canonical device tensors ([d_out, d_in] row-major) -> packed MlpWeights."""
    if out is None:
        out = MlpWeights(wtype, d_model, d_ff, Wg.device)
    for t in (Wg, Wu, Wd, Sg, Su, Sd):
        assert t is None or (t.is_cuda and t.is_contiguous())
    ctx.check(_lib.dip_pack_weights(ctx.handle, wtype, d_model, d_ff, _ptr(Wg), _ptr(Wu), _ptr(Wd),
                                    _ptr(Sg), _ptr(Su), _ptr(Sd), C.byref(out.struct), _stream()))
    return out


def dip_mask_topk(ctx: Context, x: torch.Tensor, k: int, mask_bits: Optional[torch.Tensor],
                  kept_idx: Optional[torch.Tensor]) -> None:
    batch, d = (1, x.numel()) if x.dim() == 1 else x.shape
    ctx.check(_lib.dip_mask_topk(ctx.handle, _ptr(x), batch, d, int(k), _ptr(mask_bits), _ptr(kept_idx),
                                 _stream()))


def dip_ca_mask(ctx: Context, x: torch.Tensor, k: int, gamma: float, st: CacheState,
                mask_bits: Optional[torch.Tensor], kept_idx: Optional[torch.Tensor]) -> None:
    ctx.check(_lib.dip_ca_mask(ctx.handle, _ptr(x), x.numel(), int(k), float(gamma), C.byref(st.struct),
                               _ptr(mask_bits), _ptr(kept_idx), _stream()))


def dip_sparse_gemv_gate_up(ctx: Context, w: MlpWeights, x: torch.Tensor, kept_idx: torch.Tensor, n_kept: int,
                            mask_bits: Optional[torch.Tensor], h: torch.Tensor) -> None:
    batch = 1 if x.dim() == 1 else x.shape[0]
    ctx.check(_lib.dip_sparse_gemv_gate_up(ctx.handle, C.byref(w.struct), _ptr(x), batch, _ptr(kept_idx),
                                           int(n_kept), _ptr(mask_bits), _ptr(h), _stream()))


def dip_sparse_gemv_down(ctx: Context, w: MlpWeights, h: torch.Tensor, kept_idx: torch.Tensor, n_kept: int,
                         mask_bits: Optional[torch.Tensor], y: torch.Tensor) -> None:
    batch = 1 if h.dim() == 1 else h.shape[0]
    ctx.check(_lib.dip_sparse_gemv_down(ctx.handle, C.byref(w.struct), _ptr(h), batch, _ptr(kept_idx),
                                        int(n_kept), _ptr(mask_bits), _ptr(y), _stream()))


def dip_select_gemv_gate_up(ctx: Context, w: MlpWeights, x: torch.Tensor, k_x: int, gamma: float,
                            cache_gu: Optional[CacheState], cache_d: Optional[CacheState],
                            mask_x: torch.Tensor, h: torch.Tensor) -> None:
    ctx.check(_lib.dip_select_gemv_gate_up(ctx.handle, C.byref(w.struct), _ptr(x), int(k_x), float(gamma),
                                           C.byref(cache_gu.struct) if cache_gu else None,
                                           C.byref(cache_d.struct) if cache_d else None,
                                           _ptr(mask_x), _ptr(h), _stream()))


def dip_select_gemv_down(ctx: Context, w: MlpWeights, h: torch.Tensor, k_h: int, gamma: float,
                         cache_d: Optional[CacheState], mask_h: torch.Tensor, y: torch.Tensor) -> None:
    ctx.check(_lib.dip_select_gemv_down(ctx.handle, C.byref(w.struct), _ptr(h), int(k_h), float(gamma),
                                        C.byref(cache_d.struct) if cache_d else None,
                                        _ptr(mask_h), _ptr(y), _stream()))


def dip_mlp_step(ctx: Context, w: MlpWeights, x: torch.Tensor, k_x: int, k_h: int, gamma: float,
                 cache_gu: Optional[CacheState], cache_d: Optional[CacheState], y: torch.Tensor,
                 mask_x=None, idx_x=None, h=None, mask_h=None, idx_h=None, union_counts=None) -> None:
    batch = 1 if x.dim() == 1 else x.shape[0]
    outs = StepOutputsStruct(_ptr(mask_x), _ptr(idx_x), _ptr(h), _ptr(mask_h), _ptr(idx_h), _ptr(union_counts))
    ctx.check(_lib.dip_mlp_step(ctx.handle, C.byref(w.struct), _ptr(x), batch, int(k_x), int(k_h), float(gamma),
                                C.byref(cache_gu.struct) if cache_gu else None,
                                C.byref(cache_d.struct) if cache_d else None,
                                _ptr(y), C.byref(outs), _stream()))


class Tier:
    """Where the columns of one masked input live: `backing` holds all d packed rows (pinned host
    memory, or a device tensor), the arena on the device holds the cache's columns.  Belongs to
    one CacheState; both start cold."""

    def __init__(self, cache: CacheState, backing: torch.Tensor, row_bytes: int, staging: int, device):
        assert backing.dtype == torch.uint8 and backing.is_contiguous()
        assert backing.numel() == cache.d * row_bytes
        assert backing.is_cuda or backing.is_pinned(), "the slow tier must be readable by the device"
        self.cache, self.backing = cache, backing
        self.d, self.capacity, self.staging, self.row_bytes = cache.d, cache.capacity, int(staging), int(row_bytes)
        words = (self.d + 31) // 32
        self.arena = torch.empty((self.capacity + self.staging) * self.row_bytes, dtype=torch.uint8, device=device)
        self.slot = torch.full((self.d,), -1, dtype=torch.int32, device=device)
        self.loc = torch.zeros(self.d, dtype=torch.int32, device=device)
        self.fetch = torch.zeros(4 + 2 * self.staging, dtype=torch.int32, device=device)
        self.split = torch.zeros(2 * words, dtype=torch.int32, device=device)
        self.counters = torch.zeros(2, dtype=torch.int64, device=device)
        self.struct = TierStruct(self.d, self.capacity, self.staging, 0, self.row_bytes, _ptr(backing),
                                 _ptr(self.arena), _ptr(self.slot), _ptr(self.loc), _ptr(self.fetch),
                                 _ptr(self.split), _ptr(self.counters))


def dip_mlp_step_tiered(ctx: Context, w: MlpWeights, tier_gu: Tier, tier_d: Tier, x: torch.Tensor,
                        k_x: int, k_h: int, gamma: float, y: torch.Tensor,
                        mask_x=None, idx_x=None, h=None, mask_h=None, idx_h=None) -> None:
    """One token through one block with both inputs' weights two-tiered; the caches are the tiers'."""
    outs = StepOutputsStruct(_ptr(mask_x), _ptr(idx_x), _ptr(h), _ptr(mask_h), _ptr(idx_h), None)
    ctx.check(_lib.dip_mlp_step_tiered(ctx.handle, C.byref(w.struct), C.byref(tier_gu.struct),
                                       C.byref(tier_d.struct), _ptr(x), int(k_x), int(k_h), float(gamma),
                                       C.byref(tier_gu.cache.struct), C.byref(tier_d.cache.struct),
                                       _ptr(y), C.byref(outs), _stream()))


class NeuronWeights:
    """Weights of one block laid out by neuron for Gate / Up pruning: gate and up as their own
    row-major [d_ff, d_model] matrices, down as [d_ff, d_model] with row j = W^d[:, j]."""

    def __init__(self, wtype: int, gate: torch.Tensor, up: torch.Tensor, down_t: torch.Tensor):
        d_ff, d_model = gate.shape
        assert up.shape == gate.shape and tuple(down_t.shape) == (d_ff, d_model)
        for t in (gate, up, down_t):
            assert t.is_cuda and t.is_contiguous()
        self.wtype, self.d_model, self.d_ff = int(wtype), int(d_model), int(d_ff)
        self.gate, self.up, self.down = gate, up, down_t
        self.struct = NeuronWeightsStruct(self.wtype, self.d_model, self.d_ff, 0, _ptr(gate), _ptr(up), _ptr(down_t))


def dip_mlp_step_neuron_pruned(ctx: Context, w: NeuronWeights, prune_by: str, x: torch.Tensor, k: int,
                               y: torch.Tensor, p=None, mask=None, idx=None, h=None) -> None:
    """Gate pruning (prune_by="gate") or Up pruning ("up") of one token through one block."""
    assert prune_by in ("gate", "up")
    ctx.check(_lib.dip_mlp_step_neuron_pruned(ctx.handle, C.byref(w.struct),
                                              PRUNE_BY_GATE if prune_by == "gate" else PRUNE_BY_UP, _ptr(x), int(k),
                                              _ptr(y), _ptr(p), _ptr(mask), _ptr(idx), _ptr(h), _stream()))


def dip_residual_rmsnorm(ctx: Context, x: torch.Tensor, y: torch.Tensor, x_next: torch.Tensor) -> None:
    batch, d = (1, x.numel()) if x.dim() == 1 else x.shape
    ctx.check(_lib.dip_residual_rmsnorm(ctx.handle, _ptr(x), _ptr(y), batch, d, _ptr(x_next), _stream()))


class Stack:
    """Host arrays naming the layers (and caches) of an MLP stack for dip_stack_step."""

    def __init__(self, layers: Sequence[MlpWeights], cache_gu: Optional[Sequence[CacheState]] = None,
                 cache_d: Optional[Sequence[CacheState]] = None):
        self.layers: List[MlpWeights] = list(layers)
        self.cache_gu = list(cache_gu) if cache_gu is not None else None
        self.cache_d = list(cache_d) if cache_d is not None else None
        n = len(self.layers)
        self.w_arr = (MlpWeightsStruct * n)(*[l.struct for l in self.layers])
        self.gu_arr = (CacheStateStruct * n)(*[c.struct for c in self.cache_gu]) if self.cache_gu else None
        self.d_arr = (CacheStateStruct * n)(*[c.struct for c in self.cache_d]) if self.cache_d else None


def dip_stack_step(ctx: Context, stack: Stack, x_in: torch.Tensor, k_x: int, k_h: int, gamma: float,
                   x_out: torch.Tensor, y_last: Optional[torch.Tensor] = None) -> None:
    batch = 1 if x_in.dim() == 1 else x_in.shape[0]
    ctx.check(_lib.dip_stack_step(ctx.handle, len(stack.layers), stack.w_arr, _ptr(x_in), batch, int(k_x),
                                  int(k_h), float(gamma), stack.gu_arr, stack.d_arr, _ptr(x_out),
                                  _ptr(y_last), _stream()))


class StackProbe:
    """Per-layer intermediates of one dip_stack_step_probed call (device tensors owned here)."""

    def __init__(self, n_layers: int, batch: int, d_model: int, d_ff: int, device):
        self.x = torch.empty((n_layers, batch, d_model), device=device)
        self.mask_x = torch.zeros((n_layers, batch, d_model // 32), dtype=torch.int32, device=device)
        self.h = torch.empty((n_layers, batch, d_ff), device=device)
        self.mask_h = torch.zeros((n_layers, batch, d_ff // 32), dtype=torch.int32, device=device)
        self.y = torch.empty((n_layers, batch, d_model), device=device)
        self.struct = StackProbeStruct(_ptr(self.x), _ptr(self.mask_x), _ptr(self.h), _ptr(self.mask_h), _ptr(self.y))


def dip_stack_step_probed(ctx: Context, stack: Stack, x_in: torch.Tensor, k_x: int, k_h: int, gamma: float,
                          x_out: torch.Tensor, probe: StackProbe) -> None:
    batch = 1 if x_in.dim() == 1 else x_in.shape[0]
    ctx.check(_lib.dip_stack_step_probed(ctx.handle, len(stack.layers), stack.w_arr, _ptr(x_in), batch, int(k_x),
                                         int(k_h), float(gamma), stack.gu_arr, stack.d_arr, _ptr(x_out),
                                         C.byref(probe.struct), _stream()))


def dip_sparse_gemv_down_noalloc(w: MlpWeights, h: torch.Tensor, kept_idx: torch.Tensor, n_kept: int,
                                 y: torch.Tensor) -> None:
    """y = W~d h without a Context and without any device allocation by the library.

    For callers that cannot let this library allocate: hosts whose memory pool is owned by a
    framework, serving loops that cannot afford the synchronisation an allocation implies, or
    processes with no free device memory left for a Context's workspace.  Scratch comes from a
    fixed ~4 MB array inside the library image, shared by every call on the device, so calls
    that overlap on the GPU race: keep them on one stream.  d_model is limited to 16384
    (ERR_WORKSPACE beyond); F32 and BF16 weights only.  The first call on a device does a
    one-off address look-up and should come before any stream capture.
    """
    st = _lib.dip_sparse_gemv_down_noalloc(C.byref(w.struct), _ptr(h), _ptr(kept_idx), int(n_kept), _ptr(y),
                                           _stream())
    if st == ERR_WORKSPACE:
        raise DipError(st, "d_model exceeds the no-allocation entry point's fixed scratch (max 16384)")
    if st != OK:
        raise DipError(st, "dip_sparse_gemv_down_noalloc")


# ---- mixtures of SwiGLU blocks, and prompts through a dense one -----------------------------------------------------------
def _refuse(what: str, *args) -> None:
    raise DipError(ERR_INVALID_ARG, what % args if args else what)


def _matrix(t, dtype, n: Optional[int], d: Optional[int], name: str, device: int) -> None:
    """t is a contiguous [n, d] tensor (None: any extent) of that type on that device.  Called several times per launch of a few
    microseconds: no message is formed unless it is needed."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype:
        _refuse("%s must be a tensor of %s", name, dtype)
    if t.get_device() != device or not t.is_contiguous():
        _refuse("%s must be contiguous and on device %d", name, device)
    s = t.shape
    if len(s) != 2 or (n is not None and s[0] != n) or (d is not None and s[1] != d):
        _refuse("%s must have the shape %s, got %s", name, (n, d), tuple(s))


def _blocks(d: int) -> int:
    return (d + FP8_BLOCK - 1) // FP8_BLOCK


_ROW_DTYPES = {W_BF16: torch.bfloat16, W_FP8_B128: torch.float8_e4m3fn}


class GroupedMatrix:
    """Matrices [n_experts, d_out, d_in] (or one [d_out, d_in]), bfloat16, or float8_e4m3fn with binary32 scales
    [n_experts, ceil(d_out / 128), ceil(d_in / 128)].  Nothing is copied: the tensors stay the caller's layout."""

    def __init__(self, values: torch.Tensor, scales: Optional[torch.Tensor] = None):
        if values.dim() == 2:
            values, scales = values[None], None if scales is None else scales[None]
        if values.dim() != 3 or values.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            _refuse("values must be [n_experts, d_out, d_in], bfloat16 or float8_e4m3fn")
        self.wtype = W_BF16 if values.dtype == torch.bfloat16 else W_FP8_B128
        self.n_experts, self.d_out, self.d_in = values.shape
        if (scales is not None) != (self.wtype == W_FP8_B128):
            _refuse("scales belong to float8_e4m3fn values, and only to them")
        if not values.is_cuda or not values.is_contiguous():
            _refuse("values must be a contiguous device tensor")
        if scales is not None:
            if (scales.dtype != torch.float32 or scales.device != values.device or not scales.is_contiguous() or
                    tuple(scales.shape) != (self.n_experts, _blocks(self.d_out), _blocks(self.d_in))):
                _refuse("scales must be contiguous float32 [n_experts, ceil(d_out / 128), ceil(d_in / 128)] beside the values")
        self.values, self.scales, self.device = values, scales, values.get_device()
        self.struct = GroupedMatrixStruct(self.wtype, self.n_experts, self.d_out, self.d_in, _ptr(values), _ptr(scales))
        self.ref = C.byref(self.struct)


class Rows:
    """Up to max_rows rows of d values as a grouped product takes them: bfloat16, or e4m3 codes with scales.
    n_rows of them are in use (what the last call that wrote them wrote)."""

    def __init__(self, max_rows: int, d: int, wtype: int, device):
        if wtype not in _ROW_DTYPES:
            _refuse("rows are W_BF16 or W_FP8_B128")
        self._set(torch.empty((max_rows, d), dtype=_ROW_DTYPES[wtype], device=device),
                  torch.empty((max_rows, _blocks(d)), device=device) if wtype == W_FP8_B128 else None)

    @classmethod
    def of(cls, values: torch.Tensor, scales: Optional[torch.Tensor] = None) -> "Rows":
        """Rows that are there already: all of `values` is in use."""
        if values.dim() != 2 or values.dtype not in _ROW_DTYPES.values() or not values.is_cuda or not values.is_contiguous():
            _refuse("rows are a contiguous bfloat16 or float8_e4m3fn device tensor [n, d]")
        if (scales is not None) != (values.dtype == torch.float8_e4m3fn):
            _refuse("scales belong to float8_e4m3fn rows, and only to them")
        if scales is not None:
            _matrix(scales, torch.float32, values.shape[0], _blocks(values.shape[1]), "scales", values.get_device())
        self = cls.__new__(cls)
        self._set(values, scales)
        self.n_rows = values.shape[0]
        return self

    def _set(self, values, scales):
        self.values, self.scales = values, scales
        self.max_rows, self.d = values.shape
        self.wtype = W_BF16 if scales is None else W_FP8_B128
        self.n_rows = 0
        self.device, self.ptr, self.scales_ptr = values.get_device(), _ptr(values), _ptr(scales)


class ExpertRoute:
    """A router's decisions for up to max_tokens tokens (device tensors owned here).  After a call with n tokens the
    first n rows of expert, weight and token_row, all of offset and the first offset[-1] entries of row_token are its."""

    def __init__(self, max_tokens: int, n_experts: int, top_k: int, device):
        if not 1 <= max_tokens <= MAX_TOKENS:
            _refuse("1 .. %d tokens", MAX_TOKENS)
        if not (1 <= n_experts <= MAX_EXPERTS and 1 <= top_k <= min(n_experts, MAX_TOP_K)):
            _refuse("1 .. %d experts, of which 1 .. %d are chosen", MAX_EXPERTS, MAX_TOP_K)
        self.max_tokens, self.n_experts, self.top_k = int(max_tokens), int(n_experts), int(top_k)
        ints = dict(dtype=torch.int32, device=device)
        self.expert = torch.full((max_tokens, top_k), -1, **ints)
        self.weight = torch.zeros((max_tokens, top_k), device=device)
        self.offset = torch.zeros(n_experts + 1, **ints)
        self.row_token = torch.zeros(max_tokens * top_k, **ints)
        self.token_row = torch.full((max_tokens, top_k), -1, **ints)
        self.device = self.offset.get_device()
        self.struct = ExpertRouteStruct(0, self.n_experts, self.top_k, 0, _ptr(self.expert), _ptr(self.weight), _ptr(self.offset),
                                        _ptr(self.row_token), _ptr(self.token_row))
        self.ref = C.byref(self.struct)

    @property
    def n_tokens(self) -> int:
        return self.struct.n_tokens

    @property
    def n_rows(self) -> int:
        """Most rows that the last call's tokens can have."""
        return self.struct.n_tokens * self.top_k


class ExpertWeights:
    """gate, up [n_experts, d_ff, d_model] and down [n_experts, d_model, d_ff] of a mixture (or of one dense block)."""

    def __init__(self, gate: GroupedMatrix, up: GroupedMatrix, down: GroupedMatrix):
        shape = lambda m: (m.wtype, m.n_experts, m.d_out, m.d_in, m.device)  # noqa: E731
        if not shape(gate) == shape(up) == (down.wtype, down.n_experts, down.d_in, down.d_out, down.device):
            _refuse("gate and up must be alike, and down their transposed shape")
        self.gate, self.up, self.down, self.device = gate, up, down, gate.device
        self.wtype, self.n_experts, self.d_model, self.d_ff = gate.wtype, gate.n_experts, gate.d_in, gate.d_out


class ExpertWork:
    """The buffers that dip_expert_mlp needs for up to max_tokens tokens; top_k = 0: without a route."""

    def __init__(self, max_tokens: int, top_k: int, w: ExpertWeights, device):
        if not (1 <= max_tokens <= MAX_TOKENS and 0 <= top_k <= MAX_TOP_K):
            _refuse("1 .. %d tokens, top_k 0 .. %d", MAX_TOKENS, MAX_TOP_K)
        self.max_rows, self.routed = int(max_tokens) * max(1, int(top_k)), top_k > 0
        self.wtype, self.d_model, self.d_ff = w.wtype, w.d_model, w.d_ff
        fp8 = w.wtype == W_FP8_B128
        self.rows = Rows(self.max_rows, w.d_model, w.wtype, device) if fp8 or self.routed else None
        self.h = Rows(self.max_rows, w.d_ff, w.wtype, device)
        self.out = torch.empty((self.max_rows, w.d_model), device=device) if self.routed else None
        self.device = self.h.device
        self.struct = ExpertWorkStruct(self.rows.ptr if self.rows else None, self.rows.scales_ptr if self.rows else None,
                                       self.h.ptr, self.h.scales_ptr, _ptr(self.out))
        self.ref = C.byref(self.struct)


def dip_route_experts(ctx: Context, logits: torch.Tensor, route: ExpertRoute, renormalize: bool = True) -> None:
    """logits [n, n_experts], binary32 or bfloat16, n <= route.max_tokens."""
    bf16 = isinstance(logits, torch.Tensor) and logits.dtype is torch.bfloat16
    _matrix(logits, torch.bfloat16 if bf16 else torch.float32, None, route.n_experts, "logits", ctx.device)
    n = logits.shape[0]
    if not 1 <= n <= route.max_tokens:
        _refuse("the route holds 1 .. %d tokens", route.max_tokens)
    if route.device != ctx.device:
        _refuse("the route is not on the context's device")
    before, route.struct.n_tokens = route.struct.n_tokens, n
    status = _lib.dip_route_experts(ctx.handle, logits.data_ptr(), bf16, bool(renormalize), route.ref, _stream())
    if status != OK:
        route.struct.n_tokens = before                       # (nothing was launched)
        ctx.check(status)


def _check_route(ctx: Context, route: Optional[ExpertRoute], n_tokens: int) -> None:
    if route is not None and (route.device != ctx.device or route.struct.n_tokens != n_tokens):
        _refuse("the route must be on the context's device and of %d tokens, it is of %d", n_tokens, route.struct.n_tokens)


def _check_offset(ctx: Context, offset: Optional[torch.Tensor], n_experts: int) -> None:
    if offset is None:
        if n_experts != 1:
            _refuse("several experts need the offsets of their groups")
    elif (offset.dtype is not torch.int32 or offset.get_device() != ctx.device or not offset.is_contiguous() or
          offset.shape != (n_experts + 1,)):
        _refuse("offset must be contiguous int32 [%d] on the context's device", n_experts + 1)


def dip_stage_rows(ctx: Context, x: torch.Tensor, rows: Rows, route: Optional[ExpertRoute] = None) -> None:
    """x [n, d] bfloat16 -> rows: x[t] for every row's token t, or x[r]; quantised if the rows are e4m3."""
    _matrix(x, torch.bfloat16, None, rows.d, "x", ctx.device)
    n_tokens = n = x.shape[0]
    if route is not None:
        _check_route(ctx, route, n_tokens)
        n *= route.top_k
    if rows.device != ctx.device or not 1 <= n <= rows.max_rows:
        _refuse("rows must be on the context's device and hold %d, they hold %d", n, rows.max_rows)
    ctx.check(_lib.dip_stage_rows(ctx.handle, x.data_ptr(), n_tokens, rows.d, route.ref if route is not None else None, rows.wtype,
                                  rows.ptr, rows.scales_ptr, _stream()))
    rows.n_rows = n


def dip_grouped_product(ctx: Context, w: GroupedMatrix, rows: Rows, y: torch.Tensor, offset: Optional[torch.Tensor] = None) -> None:
    """y [>= rows.n_rows, d_out], bfloat16 or float32; offset int32 [n_experts + 1], None: one expert."""
    if rows.device != ctx.device or w.device != ctx.device or rows.wtype != w.wtype or rows.d != w.d_in:
        _refuse("rows and weights must be on the context's device and agree in type and width")
    f32 = isinstance(y, torch.Tensor) and y.dtype is torch.float32
    _matrix(y, torch.float32 if f32 else torch.bfloat16, None, w.d_out, "y", ctx.device)
    if not 1 <= rows.n_rows <= y.shape[0]:
        _refuse("y has %d rows for %d", y.shape[0], rows.n_rows)
    _check_offset(ctx, offset, w.n_experts)
    ctx.check(_lib.dip_grouped_product(ctx.handle, w.ref, rows.ptr, rows.scales_ptr, rows.n_rows, _ptr(offset), y.data_ptr(), f32,
                                       _stream()))


def dip_grouped_gate_up(ctx: Context, gate: GroupedMatrix, up: GroupedMatrix, rows: Rows, h: Rows,
                        offset: Optional[torch.Tensor] = None) -> None:
    """h = silu(gate rows) * (up rows), rounded (and for e4m3 quantised) as the next product takes it."""
    for m in (gate, up):
        if (not rows.device == h.device == m.device == ctx.device or not rows.wtype == h.wtype == m.wtype or rows.d != m.d_in or
                h.d != m.d_out or m.n_experts != gate.n_experts):
            _refuse("rows, h and weights must be on the context's device and agree in type, width and number of experts")
    if not 1 <= rows.n_rows <= h.max_rows:
        _refuse("h has %d rows for %d", h.max_rows, rows.n_rows)
    _check_offset(ctx, offset, gate.n_experts)
    ctx.check(_lib.dip_grouped_gate_up(ctx.handle, gate.ref, up.ref, rows.ptr, rows.scales_ptr, rows.n_rows, _ptr(offset),
                                       h.ptr, h.scales_ptr, _stream()))
    h.n_rows = rows.n_rows


def dip_combine_rows(ctx: Context, rows: torch.Tensor, route: ExpertRoute, y: torch.Tensor) -> None:
    """y [n, d] bfloat16 = the weighted sums of rows [>= n * top_k, d], binary32; n the route's tokens."""
    n = route.struct.n_tokens
    if route.device != ctx.device or n < 1:
        _refuse("the route must be on the context's device and have tokens")
    _matrix(y, torch.bfloat16, n, None, "y", ctx.device)
    _matrix(rows, torch.float32, None, y.shape[1], "rows", ctx.device)
    if rows.shape[0] < n * route.top_k:
        _refuse("rows has %d rows for %d", rows.shape[0], n * route.top_k)
    ctx.check(_lib.dip_combine_rows(ctx.handle, rows.data_ptr(), route.ref, y.shape[1], y.data_ptr(), _stream()))


def dip_expert_mlp(ctx: Context, w: ExpertWeights, x: torch.Tensor, work: ExpertWork, y: torch.Tensor,
                   route: Optional[ExpertRoute] = None) -> None:
    """x [n, d_model] -> y [n, d_model], bfloat16, through the mixture (route) or the one dense block (no route)."""
    _matrix(x, torch.bfloat16, None, w.d_model, "x", ctx.device)
    n_tokens = n = x.shape[0]
    _matrix(y, torch.bfloat16, n_tokens, w.d_model, "y", ctx.device)
    if w.device != ctx.device or (work.wtype, work.d_model, work.d_ff, work.device) != (w.wtype, w.d_model, w.d_ff, ctx.device):
        _refuse("weights and buffers must be on the context's device, and of one shape and type")
    if route is None:
        if w.n_experts != 1:
            _refuse("several experts need a route")
    else:
        _check_route(ctx, route, n_tokens)
        if route.n_experts != w.n_experts:
            _refuse("route and weights differ in their number of experts")
        n *= route.top_k
    if work.routed != (route is not None) or not 1 <= n <= work.max_rows:
        _refuse("buffers for %d rows %s a route, %d are needed", work.max_rows, "with" if work.routed else "without", n)
    ctx.check(_lib.dip_expert_mlp(ctx.handle, w.gate.ref, w.up.ref, w.down.ref, x.data_ptr(), n_tokens,
                                  route.ref if route is not None else None, work.ref, y.data_ptr(), _stream()))
