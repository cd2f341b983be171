"""Thin ctypes binding over libr3_b200.so (the C ABI declared in include/r3.h).

Argument marshalling only: every step of the replayed layer runs in the CUDA library.  PyTorch
supplies device memory and the current stream.  There is no CPU fallback: importing this module
without a built library raises, and every call requires CUDA tensors.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
import os

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libr3_b200.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(
        f"{_LIB_PATH} is missing: build it with `python -m paper_2510_11370_b200.build` "
        "(needs nvcc; there is no CPU fallback)")
lib = ctypes.CDLL(_LIB_PATH)

R3_OK = 0
R3_ERR_INVALID_ARG, R3_ERR_UNSUPPORTED, R3_ERR_WORKSPACE, R3_ERR_CUDA = 1, 2, 3, 4
R3_ERR_SCRATCH_LIMIT = 5
R3_ERR_OUT_OF_PAGES = 6
R3_F32, R3_BF16 = 0, 1
R3_IDX_U8, R3_IDX_I16 = 1, 2
R3_GATE_NONE, R3_GATE_CHANNEL, R3_GATE_TOKEN, R3_GATE_FULL = 0, 1, 2, 3
DEV_OK, DEV_BAD_INDEX, DEV_DUP_INDEX, DEV_TIMEOUT = 0, 1, 2, 3

EXPORTS = [
    "r3_status_string", "r3_capture_topk", "r3_capture_topk_batched",
    "r3_capture_topk_workspace_bytes", "r3_capture_topk_ws", "r3_replay_gate_fwd",
    "r3_replay_gate_bwd", "r3_permute_workspace_bytes", "r3_permute", "r3_permute_static",
    "r3_grouped_swiglu_workspace_bytes", "r3_grouped_swiglu", "r3_grouped_swiglu_gather",
    "r3_expert_up_swiglu",
    "r3_expert_down", "r3_combine",
    "r3_combine_residual", "r3_combine_bwd_gates", "r3_replay_finish",
    "r3_replay_layer_workspace_bytes",
    "r3_replay_layer", "r3_replay_blocks", "r3_replay_stack_workspace_bytes", "r3_replay_stack",
    "r3_replay_layer_host_workspace_bytes", "r3_replay_layer_host", "r3_replay_layer_host_enqueue",
    "r3_replay_layer_host_chunks",
    "r3_replay_layer_same_record",
    "r3_adamw_step", "r3_normed_stack_workspace_bytes", "r3_normed_stack",
    "r3_normed_stack_train_workspace_bytes", "r3_normed_stack_train",
    "r3_norm_residual", "r3_norm_residual_bwd_workspace_bytes", "r3_norm_residual_bwd",
    "r3_token_logprobs", "r3_token_logprobs_bwd",
    "r3_prob_discrepancy_workspace_bytes", "r3_prob_discrepancy", "r3_record_diff",
    "r3_sequence_diff", "r3_grouped_swiglu_bwd_workspace_bytes", "r3_grouped_swiglu_bwd_input",
    "r3_grouped_swiglu_bwd", "r3_grouped_swiglu_train", "r3_scale_rows", "r3_input_grad_finish",
    "r3_replay_layer_train_workspace_bytes", "r3_replay_layer_train",
    "r3_replay_stack_train_workspace_bytes", "r3_replay_stack_train",
    "r3_ep_regroup_map", "r3_ep_move_rows", "r3_ep_dest_table", "r3_ep_dispatch_rows",
    "r3_ep_slot_rows", "r3_replay_finish_rows",
    "r3_record_page_bytes", "r3_record_append", "r3_record_gather",
    "r3_pagepool_create", "r3_pagepool_destroy", "r3_pagepool_free_pages", "r3_pagepool_match",
    "r3_pagepool_alloc", "r3_pagepool_publish", "r3_pagepool_release",
    "r3_selftest_bounded_wait",
]


class Shape(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("d", ctypes.c_int32), ("E", ctypes.c_int32),
                ("K", ctypes.c_int32), ("F", ctypes.c_int32), ("act_dtype", ctypes.c_int32),
                ("router_w_dtype", ctypes.c_int32), ("idx_type", ctypes.c_int32)]


class Logits(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("V", ctypes.c_int32), ("ld", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("id_bytes", ctypes.c_int32),
                ("temperature", ctypes.c_double)]


class Norm(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("d", ctypes.c_int32), ("act_dtype", ctypes.c_int32),
                ("w_dtype", ctypes.c_int32), ("gate_kind", ctypes.c_int32),
                ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
                ("branch_scale", ctypes.c_float)]


class BlockNorms(ctypes.Structure):
    _fields_ = [("w_pre", ctypes.c_void_p), ("w_post", ctypes.c_void_p), ("gate", ctypes.c_void_p),
                ("dw_pre", ctypes.c_void_p), ("dw_post", ctypes.c_void_p), ("dgate", ctypes.c_void_p),
                ("w_dtype", ctypes.c_int32), ("eps", ctypes.c_float),
                ("residual_scale", ctypes.c_float), ("branch_scale", ctypes.c_float)]


class AdamWTensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("master", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("exp_avg", ctypes.c_void_p), ("exp_avg_sq", ctypes.c_void_p),
                ("exp_avg_scale", ctypes.c_void_p), ("exp_avg_sq_scale", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("weight_decay", ctypes.c_float)]


class AdamWConfig(ctypes.Structure):
    _fields_ = [("param_dtype", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
                ("master", ctypes.c_int32), ("state_bits", ctypes.c_int32), ("step", ctypes.c_int64),
                ("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double)]


_P = ctypes.c_void_p
_SP = ctypes.POINTER(Shape)
lib.r3_status_string.restype = ctypes.c_char_p
lib.r3_status_string.argtypes = [ctypes.c_int]
lib.r3_grouped_swiglu_bwd_input.argtypes = [_SP] + [_P] * 9 + [ctypes.c_size_t, _P, _P]
lib.r3_grouped_swiglu_train.argtypes = [_SP] + [_P] * 9 + [ctypes.c_size_t, _P, _P]
lib.r3_scale_rows.argtypes = [_SP] + [_P] * 5
lib.r3_input_grad_finish.argtypes = [_SP] + [_P] * 12
lib.r3_replay_layer_train.argtypes = [_SP] + [_P] * 15 + [ctypes.c_size_t, _P, _P]
lib.r3_replay_stack_train_workspace_bytes.restype = ctypes.c_size_t
lib.r3_replay_stack_train_workspace_bytes.argtypes = [_SP, ctypes.c_int32]
lib.r3_replay_stack_train.argtypes = [_SP, ctypes.c_int32] + [_P] * 15 + [ctypes.c_size_t, _P, _P]
lib.r3_ep_regroup_map.argtypes = [_P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _P, _P, _P, _P]
lib.r3_ep_dest_table.argtypes = [_P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, _P, _P, _P]
lib.r3_ep_dispatch_rows.argtypes = [_SP, ctypes.c_int32, _P, _P, _P, _P, _P, _P, ctypes.c_int64,
                                    _P, _P]
lib.r3_ep_slot_rows.argtypes = [_SP, ctypes.c_int32, _P, _P, _P, _P, _P, ctypes.c_int64, _P, _P, _P]
lib.r3_replay_finish_rows.argtypes = [_SP] + [_P] * 10
lib.r3_ep_move_rows.argtypes = [_P, _P, _P, ctypes.c_int32, ctypes.c_size_t, ctypes.c_int32, _P]
lib.r3_grouped_swiglu_bwd.argtypes = [_SP] + [_P] * 13 + [ctypes.c_size_t, _P, _P]
for _n in ("r3_permute_workspace_bytes", "r3_grouped_swiglu_workspace_bytes",
           "r3_grouped_swiglu_bwd_workspace_bytes", "r3_replay_layer_train_workspace_bytes",
           "r3_replay_stack_workspace_bytes",
           "r3_replay_layer_workspace_bytes", "r3_replay_layer_host_workspace_bytes"):
    getattr(lib, _n).restype = ctypes.c_size_t
    getattr(lib, _n).argtypes = [_SP]
lib.r3_capture_topk.argtypes = [_SP, _P, _P, _P, _P, _P]
lib.r3_capture_topk_batched.argtypes = [_SP, ctypes.c_int32, _P, _P, _P, _P, _P]
lib.r3_capture_topk_workspace_bytes.restype = ctypes.c_size_t
lib.r3_capture_topk_workspace_bytes.argtypes = [_SP, ctypes.c_int32]
lib.r3_capture_topk_ws.argtypes = [_SP, ctypes.c_int32, _P, _P, _P, _P, _P, ctypes.c_size_t, _P]
lib.r3_replay_gate_fwd.argtypes = [_SP, _P, _P, _P, _P, _P]
lib.r3_replay_gate_bwd.argtypes = [_SP, _P, _P, _P, _P, _P]
lib.r3_permute.argtypes = [_SP, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P, _P]
lib.r3_permute_static.argtypes = [_SP, _P, _P, _P, _P, _P, _P, _P, _P, _P]
lib.r3_grouped_swiglu.argtypes = [_SP, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P, _P]
lib.r3_grouped_swiglu_gather.argtypes = [_SP, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P, _P]
lib.r3_expert_up_swiglu.argtypes = [_SP, _P, _P, _P, _P, _P, ctypes.c_size_t, _P, _P]
lib.r3_expert_down.argtypes = [_SP, _P, _P, _P, ctypes.c_size_t, _P, _P]
lib.r3_combine.argtypes = [_SP, _P, _P, _P, _P, _P]
lib.r3_combine_residual.argtypes = [_SP, _P, _P, _P, _P, _P, _P]
lib.r3_replay_blocks.argtypes = [_SP, ctypes.c_int32] + [_P] * 10 + [ctypes.c_size_t, _P, _P]
lib.r3_replay_stack.argtypes = [_SP, ctypes.c_int32] + [_P] * 10 + [ctypes.c_size_t, _P, _P]
lib.r3_combine_bwd_gates.argtypes = [_SP, _P, _P, _P, _P, _P]
lib.r3_replay_finish.argtypes = [_SP] + [_P] * 11
lib.r3_replay_layer.argtypes = [_SP] + [_P] * 11 + [ctypes.c_size_t, _P, _P]
lib.r3_replay_layer_same_record.argtypes = [_SP] + [_P] * 11 + [ctypes.c_size_t, _P, _P]
lib.r3_replay_layer_host.argtypes = [_SP] + [_P] * 10 + [ctypes.c_size_t, _P, _P]
lib.r3_replay_layer_host_enqueue.argtypes = [_SP] + [_P] * 10 + [ctypes.c_size_t, _P, _P]
_BN = ctypes.POINTER(BlockNorms)
lib.r3_normed_stack_workspace_bytes.restype = ctypes.c_size_t
lib.r3_normed_stack_workspace_bytes.argtypes = [_SP]
lib.r3_normed_stack.argtypes = [_SP, ctypes.c_int32, _BN] + [_P] * 8 + [ctypes.c_size_t, _P, _P]
lib.r3_normed_stack_train_workspace_bytes.restype = ctypes.c_size_t
lib.r3_normed_stack_train_workspace_bytes.argtypes = [_SP, ctypes.c_int32]
lib.r3_normed_stack_train.argtypes = ([_SP, ctypes.c_int32, _BN] + [_P] * 19
                                      + [ctypes.c_size_t, _P, _P])
lib.r3_adamw_step.argtypes = [ctypes.POINTER(AdamWConfig), _P, ctypes.c_int32, _P, _P, _P]
_NP = ctypes.POINTER(Norm)
lib.r3_norm_residual.argtypes = [_NP] + [_P] * 8
lib.r3_norm_residual_bwd_workspace_bytes.restype = ctypes.c_size_t
lib.r3_norm_residual_bwd_workspace_bytes.argtypes = [_NP]
lib.r3_norm_residual_bwd.argtypes = [_NP] + [_P] * 13 + [ctypes.c_size_t, _P]
lib.r3_token_logprobs.argtypes = [ctypes.POINTER(Logits)] + [_P] * 5 + [ctypes.c_int32] + [_P] * 4
lib.r3_token_logprobs_bwd.argtypes = ([ctypes.POINTER(Logits)] + [_P] * 7 + [ctypes.c_int64]
                                      + [_P] * 2)
lib.r3_prob_discrepancy_workspace_bytes.restype = ctypes.c_size_t
lib.r3_prob_discrepancy_workspace_bytes.argtypes = [ctypes.c_int64]
lib.r3_prob_discrepancy.argtypes = [_P, _P, ctypes.c_int64, _P, ctypes.c_int32, _P, _P, _P,
                                    ctypes.c_size_t, _P]
lib.r3_record_diff.argtypes = [_SP, ctypes.c_int32, _P, _P, _P, _P, _P, _P, _P]
lib.r3_sequence_diff.argtypes = [_P, _P, ctypes.c_int32, _P, _P]
_I32 = ctypes.c_int32
lib.r3_record_page_bytes.restype = ctypes.c_size_t
lib.r3_record_page_bytes.argtypes = [_SP, _I32, _I32]
lib.r3_record_append.argtypes = [_SP, _I32, _I32, _I32, _P, _P, _I32, _P, _P, _I32, _P, _I32, _P, _P]
lib.r3_record_gather.argtypes = [_SP, _I32, _I32, _I32, _P, _P, _I32, _P, _I32, _P, _I32, _P, _P]
lib.r3_pagepool_create.restype = ctypes.c_void_p
lib.r3_pagepool_create.argtypes = [_I32, _I32]
lib.r3_pagepool_destroy.restype = None
lib.r3_pagepool_destroy.argtypes = [_P]
lib.r3_pagepool_free_pages.argtypes = [_P]
lib.r3_pagepool_match.argtypes = [_P, _P, _I32, _P, _I32]
lib.r3_pagepool_alloc.argtypes = [_P, _I32, _P]
lib.r3_pagepool_publish.argtypes = [_P, _P, _I32, _P, _I32]
lib.r3_pagepool_release.argtypes = [_P, _P, _I32]
lib.r3_selftest_bounded_wait.argtypes = [ctypes.c_int64, _P, _P, _P]
lib.r3_replay_layer_host_chunks.argtypes = [_SP, _P]
_NOT_STATUS = ("r3_status_string", "r3_pagepool_create", "r3_pagepool_destroy",
               "r3_replay_layer_host_chunks")
for _n in EXPORTS:
    if _n not in _NOT_STATUS and not _n.endswith("_bytes"):
        getattr(lib, _n).restype = ctypes.c_int


class R3Error(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(lib.r3_status_string(code).decode())


def _check(code: int) -> None:
    if code != R3_OK:
        raise R3Error(code)


_ACT = {torch.float32: R3_F32, torch.bfloat16: R3_BF16}
_IDX = {torch.uint8: R3_IDX_U8, torch.int16: R3_IDX_I16}


def make_shape(T, d, E, K, F, act=torch.bfloat16, router=torch.float32, idx=torch.uint8) -> Shape:
    return Shape(T, d, E, K, F, _ACT[act], _ACT[router], _IDX[idx])


def shape_of(w) -> Shape:
    """Shape of a synth.Workload."""
    return make_shape(w.T, w.d, w.E, w.K, w.F, w.act_dtype, w.router_dtype, w.idx_dtype)


def _act_dtype(s: Shape):
    return torch.bfloat16 if s.act_dtype == R3_BF16 else torch.float32


def _idx_dtype(s: Shape):
    return torch.uint8 if s.idx_type == R3_IDX_U8 else torch.int16


def _ptr(t, host: bool = False):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError("expected a torch.Tensor")
    if host:
        if t.is_cuda:
            raise ValueError("expected a host tensor")
    elif not t.is_cuda:
        raise ValueError("expected a CUDA tensor (there is no CPU path)")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


# the current stream's handle without a Stream object around it (4 us less per call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                      lambda device: torch.cuda.current_stream(device).cuda_stream)


def _stream(stream=None):
    if stream is None:
        return ctypes.c_void_p(_raw_stream(torch.cuda.current_device()))
    return ctypes.c_void_p(stream.cuda_stream)


def _in_order(fn):
    """For a call that allocates and takes a stream.  With stream= another one than the current, what the
    call allocates is that stream's memory (torch.cuda.stream): scratch that goes back on return is then
    reused behind the kernels that still work on it, and new memory is free of work that the current
    stream has not finished.  New outputs are also marked as used by the stream that was current, which is
    where the caller goes on with them."""
    at = list(inspect.signature(fn).parameters).index("stream")

    @functools.wraps(fn)
    def call(*args, **kw):
        stream = args[at] if len(args) > at else kw.get("stream")
        if stream is None:
            return fn(*args, **kw)
        caller = torch.cuda.current_stream(stream.device)
        with torch.cuda.stream(stream):
            out = fn(*args, **kw)
        if stream != caller:
            given = {id(a) for a in (*args, *kw.values())}
            for t in out if isinstance(out, tuple) else (out,):
                if isinstance(t, torch.Tensor) and id(t) not in given:
                    t.record_stream(caller)
        return out
    return call


def _dev(*ts):
    for t in ts:
        if isinstance(t, torch.Tensor):
            return t.device
    return torch.device("cuda")


def workspace(nbytes: int, device) -> torch.Tensor:
    """Device scratch of at least nbytes, 256-byte aligned (torch's allocator aligns to 512)."""
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _scratch(ws, nbytes: int, dev) -> torch.Tensor:
    """A call's scratch: the caller's, checked, or new."""
    if ws is None:
        return workspace(nbytes, dev)
    if not isinstance(ws, torch.Tensor):
        raise TypeError("ws: expected a torch.Tensor")
    if ws.device != dev:
        raise ValueError(f"ws: on {ws.device}, expected {dev}")
    if not ws.is_contiguous():
        raise ValueError("ws: tensor must be contiguous")
    return ws


def new_status(device) -> torch.Tensor:
    return torch.zeros(1, dtype=torch.int32, device=device)


# ---------------------------------------------------------------------------------------------
@_in_order
def capture_topk(s: Shape, x, w_router, idx_out=None, logits_out=None, *, want_idx=True,
                 want_logits=False, stream=None):
    """Router logits + TopKMask.  Returns (idx [T,K] or None, logits [T,E] or None)."""
    dev = _dev(x)
    if idx_out is None and want_idx:
        idx_out = torch.empty((s.T, s.K), dtype=_idx_dtype(s), device=dev)
    if logits_out is None and want_logits:
        logits_out = torch.empty((s.T, s.E), dtype=torch.float32, device=dev)
    _check(lib.r3_capture_topk(ctypes.byref(s), _ptr(x), _ptr(w_router), _ptr(idx_out),
                               _ptr(logits_out), _stream(stream)))
    return idx_out, logits_out


@_in_order
def capture_topk_batched(s: Shape, L: int, x, w_router, idx_out=None, logits_out=None, *,
                         want_idx=True, want_logits=False, stream=None):
    """L layers at once: x [L,T,d], w_router [L,E,d] -> idx [L,T,K], logits [L,T,E]."""
    dev = _dev(x)
    if idx_out is None and want_idx:
        idx_out = torch.empty((L, s.T, s.K), dtype=_idx_dtype(s), device=dev)
    if logits_out is None and want_logits:
        logits_out = torch.empty((L, s.T, s.E), dtype=torch.float32, device=dev)
    _check(lib.r3_capture_topk_batched(ctypes.byref(s), L, _ptr(x), _ptr(w_router),
                                       _ptr(idx_out), _ptr(logits_out), _stream(stream)))
    return idx_out, logits_out


def capture_topk_workspace_bytes(s: Shape, L: int = 1) -> int:
    return lib.r3_capture_topk_workspace_bytes(ctypes.byref(s), L)


@_in_order
def capture_topk_ws(s: Shape, L: int, x, w_router, idx_out=None, logits_out=None, *, ws=None,
                    want_idx=True, want_logits=False, stream=None):
    """capture_topk with scratch, so that float32 router weights run on the tensor cores too."""
    dev = _dev(x)
    lead = (L,) if x.dim() == 3 else ()
    if idx_out is None and want_idx:
        idx_out = torch.empty(lead + (s.T, s.K), dtype=_idx_dtype(s), device=dev)
    if logits_out is None and want_logits:
        logits_out = torch.empty(lead + (s.T, s.E), dtype=torch.float32, device=dev)
    if ws is None:
        ws = workspace(capture_topk_workspace_bytes(s, L), dev)
    _check(lib.r3_capture_topk_ws(ctypes.byref(s), L, _ptr(x), _ptr(w_router), _ptr(idx_out),
                                  _ptr(logits_out), _ptr(ws), ws.numel(), _stream(stream)))
    return idx_out, logits_out


@_in_order
def replay_gate_fwd(s: Shape, logits, idx, gates=None, dev_status=None, stream=None):
    if gates is None:
        gates = torch.empty((s.T, s.K), dtype=torch.float32, device=_dev(logits))
    _check(lib.r3_replay_gate_fwd(ctypes.byref(s), _ptr(logits), _ptr(idx), _ptr(gates),
                                  _ptr(dev_status), _stream(stream)))
    return gates


@_in_order
def replay_gate_bwd(s: Shape, gates, dgates, idx, dlogits=None, stream=None):
    if dlogits is None:
        dlogits = torch.empty((s.T, s.E), dtype=torch.float32, device=_dev(gates))
    _check(lib.r3_replay_gate_bwd(ctypes.byref(s), _ptr(gates), _ptr(dgates), _ptr(idx),
                                  _ptr(dlogits), _stream(stream)))
    return dlogits


def permute_workspace_bytes(s: Shape) -> int:
    return lib.r3_permute_workspace_bytes(ctypes.byref(s))


@_in_order
def permute(s: Shape, idx, x=None, *, out=None, ws=None, dev_status=None, stream=None):
    """Returns (counts, offsets, row_of_slot, slot_of_row, xp or None)."""
    dev = _dev(idx)
    R = s.T * s.K
    if out is None:
        counts = torch.empty(s.E, dtype=torch.int32, device=dev)
        offsets = torch.empty(s.E + 1, dtype=torch.int32, device=dev)
        ros = torch.empty((s.T, s.K), dtype=torch.int32, device=dev)
        sor = torch.empty(R, dtype=torch.int32, device=dev)
        xp = torch.empty((R, s.d), dtype=_act_dtype(s), device=dev) if x is not None else None
    else:
        counts, offsets, ros, sor, xp = out
    if ws is None:
        ws = workspace(permute_workspace_bytes(s), dev)
    _check(lib.r3_permute(ctypes.byref(s), _ptr(idx), _ptr(x), _ptr(counts), _ptr(offsets),
                          _ptr(ros), _ptr(sor), _ptr(xp), _ptr(ws), ws.numel(),
                          _ptr(dev_status), _stream(stream)))
    return counts, offsets, ros, sor, xp


def permute_static(s: Shape, idx, x, counts, offsets, row_of_slot, slot_of_row, xp, *,
                   dev_status=None, stream=None):
    """r3_permute with the scratch inside the library: for callers that cannot allocate device
    memory where they call from (their memory belongs to someone else's pool, or was budgeted
    ahead of time).  All outputs are passed in; nothing is allocated here either.  Raises
    R3Error(R3_ERR_SCRATCH_LIMIT) when E * ceil(T / 256) > 262144.  Do not overlap calls."""
    _check(lib.r3_permute_static(ctypes.byref(s), _ptr(idx), _ptr(x), _ptr(counts),
                                 _ptr(offsets), _ptr(row_of_slot), _ptr(slot_of_row), _ptr(xp),
                                 _ptr(dev_status), _stream(stream)))
    return counts, offsets, row_of_slot, slot_of_row, xp


def grouped_swiglu_workspace_bytes(s: Shape) -> int:
    return lib.r3_grouped_swiglu_workspace_bytes(ctypes.byref(s))


@_in_order
def grouped_swiglu(s: Shape, xp, offsets, w_gate, w_up, w_down, o=None, *, ws=None,
                   dev_status=None, stream=None):
    dev = _dev(xp)
    if o is None:
        o = torch.empty((s.T * s.K, s.d), dtype=_act_dtype(s), device=dev)
    if ws is None:
        ws = workspace(grouped_swiglu_workspace_bytes(s), dev)
    _check(lib.r3_grouped_swiglu(ctypes.byref(s), _ptr(xp), _ptr(offsets), _ptr(w_gate),
                                 _ptr(w_up), _ptr(w_down), _ptr(o), _ptr(ws), ws.numel(),
                                 _ptr(dev_status), _stream(stream)))
    return o


@_in_order
def grouped_swiglu_gather(s: Shape, x, slot_of_row, offsets, w_gate, w_up, w_down, o=None, *,
                          ws=None, dev_status=None, stream=None):
    """grouped_swiglu reading the token rows in place from x [T,d] through slot_of_row (bf16)."""
    dev = _dev(x)
    if o is None:
        o = torch.empty((s.T * s.K, s.d), dtype=_act_dtype(s), device=dev)
    if ws is None:
        ws = workspace(grouped_swiglu_workspace_bytes(s), dev)
    _check(lib.r3_grouped_swiglu_gather(ctypes.byref(s), _ptr(x), _ptr(slot_of_row), _ptr(offsets),
                                        _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(o), _ptr(ws),
                                        ws.numel(), _ptr(dev_status), _stream(stream)))
    return o


def expert_up_swiglu(s: Shape, xp, offsets, w_gate, w_up, ws, dev_status=None, stream=None):
    """First half of grouped_swiglu: tile list + h = silu(xp Wg^T) * (xp Wu^T) into `ws`."""
    _check(lib.r3_expert_up_swiglu(ctypes.byref(s), _ptr(xp), _ptr(offsets), _ptr(w_gate),
                                   _ptr(w_up), _ptr(ws), ws.numel(), _ptr(dev_status),
                                   _stream(stream)))


def expert_down(s: Shape, w_down, o, ws, dev_status=None, stream=None):
    """Second half of grouped_swiglu: o = h W_down^T with h taken from `ws`."""
    _check(lib.r3_expert_down(ctypes.byref(s), _ptr(w_down), _ptr(o), _ptr(ws), ws.numel(),
                              _ptr(dev_status), _stream(stream)))
    return o


@_in_order
def combine(s: Shape, o, row_of_slot, gates, y=None, stream=None):
    if y is None:
        y = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=_dev(o))
    _check(lib.r3_combine(ctypes.byref(s), _ptr(o), _ptr(row_of_slot), _ptr(gates), _ptr(y),
                          _stream(stream)))
    return y


@_in_order
def combine_residual(s: Shape, o, row_of_slot, gates, residual, y=None, stream=None):
    """y = residual + sum_j gates[:, j] * o[row_of_slot[:, j]]."""
    if y is None:
        y = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=_dev(o))
    _check(lib.r3_combine_residual(ctypes.byref(s), _ptr(o), _ptr(row_of_slot), _ptr(gates),
                                   _ptr(residual), _ptr(y), _stream(stream)))
    return y


@_in_order
def replay_blocks(s: Shape, L: int, x, w_router, idx, w_gate, w_up, w_down, dy, *, y=None,
                  dlogits=None, ws=None, dev_status=None, stream=None):
    """L independent replayed blocks, all tensors stacked on a leading layer axis.
    Returns (y [L,T,d], dlogits [L,T,E])."""
    dev = _dev(x)
    if y is None:
        y = torch.empty((L, s.T, s.d), dtype=_act_dtype(s), device=dev)
    if dlogits is None:
        dlogits = torch.empty((L, s.T, s.E), dtype=torch.float32, device=dev)
    if ws is None:
        ws = workspace(replay_layer_workspace_bytes(s), dev)
    _check(lib.r3_replay_blocks(ctypes.byref(s), L, _ptr(x), _ptr(w_router), _ptr(idx),
                                _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(dy), _ptr(y),
                                _ptr(dlogits), _ptr(ws), ws.numel(), _ptr(dev_status),
                                _stream(stream)))
    return y, dlogits


def replay_stack_workspace_bytes(s: Shape) -> int:
    return lib.r3_replay_stack_workspace_bytes(ctypes.byref(s))


@_in_order
def replay_stack(s: Shape, L: int, x0, w_router, idx, w_gate, w_up, w_down, dy, *, x_out=None,
                 dlogits=None, ws=None, dev_status=None, stream=None):
    """L residual MoE blocks with replayed routing.  Returns (x_L [T,d], dlogits [L,T,E])."""
    dev = _dev(x0)
    if x_out is None:
        x_out = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    if dlogits is None:
        dlogits = torch.empty((L, s.T, s.E), dtype=torch.float32, device=dev)
    if ws is None:
        ws = workspace(replay_stack_workspace_bytes(s), dev)
    _check(lib.r3_replay_stack(ctypes.byref(s), L, _ptr(x0), _ptr(w_router), _ptr(idx),
                               _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(dy), _ptr(x_out),
                               _ptr(dlogits), _ptr(ws), ws.numel(), _ptr(dev_status),
                               _stream(stream)))
    return x_out, dlogits


@_in_order
def combine_bwd_gates(s: Shape, dy, o, row_of_slot, dgates=None, stream=None):
    if dgates is None:
        dgates = torch.empty((s.T, s.K), dtype=torch.float32, device=_dev(o))
    _check(lib.r3_combine_bwd_gates(ctypes.byref(s), _ptr(dy), _ptr(o), _ptr(row_of_slot),
                                    _ptr(dgates), _stream(stream)))
    return dgates


@_in_order
def replay_finish(s: Shape, logits, idx, o, row_of_slot, dy, *, residual=None, y=None, gates=None,
                  dlogits=None, dev_status=None, stream=None):
    """Replay gate + combine + gate gradient + router-logit gradient in one pass over `o`
    (K <= 8).  Returns (y, gates, dlogits)."""
    dev = _dev(o)
    if y is None:
        y = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    if gates is None:
        gates = torch.empty((s.T, s.K), dtype=torch.float32, device=dev)
    if dlogits is None:
        dlogits = torch.empty((s.T, s.E), dtype=torch.float32, device=dev)
    _check(lib.r3_replay_finish(ctypes.byref(s), _ptr(logits), _ptr(idx), _ptr(o),
                                _ptr(row_of_slot), _ptr(dy), _ptr(residual), _ptr(y), _ptr(gates),
                                _ptr(dlogits), _ptr(dev_status), _stream(stream)))
    return y, gates, dlogits


def replay_layer_workspace_bytes(s: Shape) -> int:
    return lib.r3_replay_layer_workspace_bytes(ctypes.byref(s))


@_in_order
def replay_layer(s: Shape, x, w_router, idx, w_gate, w_up, w_down, dy, *, y=None, dlogits=None,
                 gates=None, ws=None, dev_status=None, stream=None):
    """Forward + router-logit backward of the replayed layer.  Returns (y, dlogits, gates)."""
    dev = _dev(x)
    if y is None:
        y = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    if dlogits is None:
        dlogits = torch.empty((s.T, s.E), dtype=torch.float32, device=dev)
    if gates is None:
        gates = torch.empty((s.T, s.K), dtype=torch.float32, device=dev)
    if ws is None:
        ws = workspace(replay_layer_workspace_bytes(s), dev)
    _check(lib.r3_replay_layer(ctypes.byref(s), _ptr(x), _ptr(w_router), _ptr(idx), _ptr(w_gate),
                               _ptr(w_up), _ptr(w_down), _ptr(dy), _ptr(y), _ptr(dlogits),
                               _ptr(gates), _ptr(ws), ws.numel(), _ptr(dev_status),
                               _stream(stream)))
    return y, dlogits, gates


@_in_order
def replay_layer_same_record(s: Shape, x, w_router, idx, w_gate, w_up, w_down, dy, *, ws, y=None,
                             dlogits=None, gates=None, dev_status=None, stream=None):
    """replay_layer for another pass over the record of the preceding replay_layer call on `ws`:
    the dispatch and the expert work lists left there are used again."""
    dev = _dev(x)
    if y is None:
        y = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    if dlogits is None:
        dlogits = torch.empty((s.T, s.E), dtype=torch.float32, device=dev)
    if gates is None:
        gates = torch.empty((s.T, s.K), dtype=torch.float32, device=dev)
    _check(lib.r3_replay_layer_same_record(ctypes.byref(s), _ptr(x), _ptr(w_router), _ptr(idx),
                                           _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(dy),
                                           _ptr(y), _ptr(dlogits), _ptr(gates), _ptr(ws),
                                           ws.numel(), _ptr(dev_status), _stream(stream)))
    return y, dlogits, gates


def replay_layer_host_workspace_bytes(s: Shape) -> int:
    return lib.r3_replay_layer_host_workspace_bytes(ctypes.byref(s))


def replay_layer_host_chunks(s: Shape) -> list:
    """Token offsets [0, ..., T] of the chunks r3_replay_layer_host sends one after the other."""
    starts = (ctypes.c_int64 * 17)()
    lib.r3_replay_layer_host_chunks.restype = ctypes.c_int32
    n = lib.r3_replay_layer_host_chunks(ctypes.byref(s), starts)
    if n <= 0:
        raise R3Error(1)
    return [int(starts[i]) for i in range(n + 1)]


def replay_layer_host(s: Shape, x_host, w_router, idx_host, w_gate, w_up, w_down, dy_host,
                      y_host, dlogits_host, *, ws, dev_status=None, stream=None):
    """As replay_layer with x, idx, dy, y, dlogits in (pinned) host memory; synchronises."""
    _check(lib.r3_replay_layer_host(ctypes.byref(s), _ptr(x_host, True), _ptr(w_router),
                                    _ptr(idx_host, True), _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                    _ptr(dy_host, True), _ptr(y_host, True),
                                    _ptr(dlogits_host, True), _ptr(ws), ws.numel(),
                                    _ptr(dev_status), _stream(stream)))
    return y_host, dlogits_host


def replay_layer_host_enqueue(s: Shape, x_host, w_router, idx_host, w_gate, w_up, w_down, dy_host,
                              y_host, dlogits_host, *, ws, dev_status=None, stream=None):
    """As replay_layer_host without the final synchronisation: the result is in y_host and
    dlogits_host once `stream` has been synchronised."""
    _check(lib.r3_replay_layer_host_enqueue(ctypes.byref(s), _ptr(x_host, True), _ptr(w_router),
                                            _ptr(idx_host, True), _ptr(w_gate), _ptr(w_up),
                                            _ptr(w_down), _ptr(dy_host, True), _ptr(y_host, True),
                                            _ptr(dlogits_host, True), _ptr(ws), ws.numel(),
                                            _ptr(dev_status), _stream(stream)))
    return y_host, dlogits_host


# ---------------------------------------------------------------------------------------------
def _expect(name: str, t, shape, dtype, device) -> None:
    """Refuses a tensor that is not what the call documents (None passes)."""
    if t is None:
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    dtypes = dtype if isinstance(dtype, tuple) else (dtype,)
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: dtype {t.dtype}, expected {' or '.join(map(str, dtypes))}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")


def _arg(name: str, t, shape, dtype, device):
    """The address of a contiguous tensor of the documented kind (None passes)."""
    if t is None:
        return None
    if type(t) not in (torch.Tensor, torch.nn.Parameter) or t.dtype != dtype or t.shape != shape \
            or t.device != device:
        _expect(name, t, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name}: tensor must be contiguous")
    return t.data_ptr()


def _device_of(name: str, t) -> torch.device:
    """The device of a call's first tensor, which has to be the current one: kernels are enqueued
    on the current device's stream."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: expected a torch.Tensor")
    if not t.is_cuda:
        raise ValueError("expected a CUDA tensor (there is no CPU path)")
    dev = t.device
    if dev.index != torch.cuda.current_device():
        raise ValueError(f"{name}: on {dev}, which is not the current device")
    return dev


_GATE_SHAPES = {"channel": (R3_GATE_CHANNEL, lambda T, d: ((d,),)),
                "token": (R3_GATE_TOKEN, lambda T, d: ((T,), (T, 1))),
                "full": (R3_GATE_FULL, lambda T, d: ((T, d),))}


def _gate_kind(gate, rows, d, w_dtype, said):
    """What a gate is broadcast along: as the caller says, or by its shape.  With as many rows as columns
    a vector may be a gate [d], of the weights' type, or a gate [T], float32: where the types leave it open
    the caller has to say."""
    shape = gate.shape
    if said is not None:
        if said not in _GATE_SHAPES:
            raise ValueError(f"gate_kind: {said!r}, expected 'channel', 'token' or 'full'")
        kind, shapes = _GATE_SHAPES[said]
        if shape in shapes(rows, d):
            return kind
        raise ValueError(f"gate: shape {tuple(shape)}, expected "
                         + " or ".join(str(list(s)) for s in shapes(rows, d)))
    if shape == (d,):
        if rows != d or gate.dtype != torch.float32:
            return R3_GATE_CHANNEL
        if w_dtype is not None and w_dtype != torch.float32:
            return R3_GATE_TOKEN
        raise ValueError(f"gate: [{d}] is one factor per channel or per token; say gate_kind='channel' or "
                         f"'token' (or pass [{d}, 1])")
    if shape == (rows, d):
        return R3_GATE_FULL
    if shape == (rows, 1) or shape == (rows,):
        return R3_GATE_TOKEN
    raise ValueError(f"gate: shape {tuple(shape)}, expected [{d}], [{rows}], [{rows}, 1] or [{rows}, {d}]")


def _norm_shape(rows, d, act, w_post, gate, w_pre, eps, residual_scale, branch_scale, dev, gate_kind=None):
    """The r3_norm of a call and the addresses of w_post, gate and w_pre, which are checked: w_post,
    w_pre and a gate [d] share one type."""
    act_code = _ACT.get(act)
    if act_code is None:
        raise ValueError(f"activations: dtype {act}, expected float32 or bfloat16")
    kind, like = R3_GATE_NONE, w_post if w_post is not None else w_pre
    if gate is not None:
        kind = _gate_kind(gate, rows, d, like.dtype if like is not None else None, gate_kind)
        if kind == R3_GATE_CHANNEL and like is None:
            like = gate
    w_dtype = like.dtype if like is not None else act
    w_code = _ACT.get(w_dtype)
    if w_code is None:
        raise ValueError(f"weights: dtype {w_dtype}, expected float32 or bfloat16")
    post = _arg("w_post", w_post, (d,), w_dtype, dev)
    pre = _arg("w_pre", w_pre, (d,), w_dtype, dev)
    if gate is not None:
        want = w_dtype if kind == R3_GATE_CHANNEL else torch.float32 if kind == R3_GATE_TOKEN else act
        gate = _arg("gate", gate, gate.shape, want, dev)
    return Norm(rows, d, act_code, w_code, kind, eps, residual_scale, branch_scale), post, gate, pre


@_in_order
def norm_residual(x, y=None, *, w_post=None, gate=None, w_pre=None, eps=1e-6, residual_scale=1.0,
                  branch_scale=1.0, gate_kind=None, x_out=None, h=None, stream=None):
    """From one residual block to the next: x_out = residual_scale x + branch_scale gate
    RMSNorm(y) w_post, h = RMSNorm(x_out) w_pre, in one pass.  x, y [T, d] float32 or bfloat16; gate
    None, [d], [T] or [T, 1] float32, or [T, d]; gate_kind ("channel", "token", "full") says which, and
    has to where T = d and a float32 vector beside float32 weights (or none) could be either.  Without y
    only h = RMSNorm(x) w_pre; without w_post the branch is not normalised; without w_pre there is no h.
    Returns (x_out, h), None for what there is not.  x_out may be x, h may be y (in place)."""
    dev = _device_of("x", x)
    shape, act = x.shape, x.dtype
    rows, d = shape
    s, post, gate, pre = _norm_shape(rows, d, act, w_post, gate, w_pre, eps, residual_scale,
                                     branch_scale, dev, gate_kind)
    src = _arg("x", x, shape, act, dev)
    if y is not None and x_out is None:
        x_out = torch.empty_like(x)
        at_x = x_out.data_ptr()
    else:
        at_x = _arg("x_out", x_out, shape, act, dev)
    if w_pre is not None and h is None:
        h = torch.empty_like(x)
        at_h = h.data_ptr()
    else:
        at_h = _arg("h", h, shape, act, dev)
    _check(lib.r3_norm_residual(ctypes.byref(s), src, _arg("y", y, shape, act, dev), post, gate, pre,
                                at_x, at_h, _stream(stream)))
    return x_out, h


@_in_order
def norm_residual_bwd(x_out, y, dx_out, dh=None, *, w_post=None, gate=None, w_pre=None, eps=1e-6,
                      residual_scale=1.0, branch_scale=1.0, gate_kind=None, dx=None, dy=None, ws=None,
                      stream=None):
    """Gradients of norm_residual from dx_out [T, d] (or None) and dh [T, d]: (dx, dy, dw_post [d],
    dgate, dw_pre [d]), None for what the call has not; dgate has the gate's shape; dw_* and the dgate of
    a gate [d], [T] or [T, 1] are float32.  x_out and y are the forward's (x_out may be None without
    w_pre)."""
    like = x_out if x_out is not None else dx_out
    dev = _device_of("x_out", like)
    shape, act = like.shape, like.dtype
    rows, d = shape
    s, post, gate_at, pre = _norm_shape(rows, d, act, w_post, gate, w_pre, eps, residual_scale,
                                        branch_scale, dev, gate_kind)
    src = [_arg(name, t, shape, act, dev) for name, t in
           (("x_out", x_out), ("y", y), ("dx_out", dx_out), ("dh", dh))]
    if dx is None:
        dx = torch.empty_like(like)
        at_dx = dx.data_ptr()
    else:
        at_dx = _arg("dx", dx, shape, act, dev)
    if y is not None and dy is None:
        dy = torch.empty_like(like)
        at_dy = dy.data_ptr()
    else:
        at_dy = _arg("dy", dy, shape, act, dev)
    # the float32 sums over tokens are the rows of one buffer (d is a multiple of 8: aligned)
    channel = s.gate_kind == R3_GATE_CHANNEL
    dw_post = dgate = dw_pre = None
    wanted = (post is not None) + channel + (pre is not None)
    if wanted:
        sums = list(like.new_empty((wanted, d), dtype=torch.float32).unbind(0))
        if post is not None:
            dw_post = sums.pop()
        if channel:
            dgate = sums.pop()
        if pre is not None:
            dw_pre = sums.pop()
    if gate is not None and not channel:
        dgate = torch.empty_like(gate)           # float32 [T] or [T, 1], or [T, d] of the rows' type
    ws = _scratch(ws, lib.r3_norm_residual_bwd_workspace_bytes(ctypes.byref(s)), dev)
    _check(lib.r3_norm_residual_bwd(
        ctypes.byref(s), src[0], src[1], post, gate_at, pre, src[2], src[3],
        at_dx, at_dy, None if dw_post is None else dw_post.data_ptr(),
        None if dgate is None else dgate.data_ptr(),
        None if dw_pre is None else dw_pre.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream)))
    return dx, dy, dw_post, dgate, dw_pre


ADAMW_BLOCK = 256        # elements that share one scale of an 8-bit state


class AdamW:
    """AdamW over a list of tensors, one launch per step (r3_adamw_step): the handle that a training
    program keeps beside its parameters.

    params, grads: lists of contiguous CUDA tensors of equal sizes, one dtype each (float32 or
    bfloat16).  masters: None, True (float32 copies of bfloat16 params are made and kept) or a list
    of float32 tensors.  States are made (zero) or given as lists: float32, or with state_bits=8
    float8_e4m3fn codes plus one float32 scale per 256 elements (exp_avg_sq then holds the root of
    the second moment).  What is made here is filled on the current stream; a first step on another one waits
    for it like for any tensor.  weight_decay: a number, or one per tensor.  The handle keeps its tensors
    memory alive (one whose .data is exchanged needs a new handle); set_grads() exchanges the gradients,
    and without any (None) the handle is one for normed_stack_train, which supplies them."""

    def __init__(self, params, grads=None, *, masters=None, exp_avg=None, exp_avg_sq=None,
                 exp_avg_scale=None, exp_avg_sq_scale=None, state_bits=32, betas=(0.9, 0.95),
                 eps=1e-8, weight_decay=0.0):
        self.params = list(params)
        if not self.params:
            raise ValueError("AdamW: no tensors")
        self._dev = _device_of("params[0]", self.params[0])
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits: {state_bits}, expected 8 or 32")
        self.state_bits = state_bits
        sizes = [p.numel() for p in self.params]
        dtype = self.params[0].dtype
        if dtype not in _ACT:
            raise ValueError(f"params: dtype {dtype}, expected float32 or bfloat16")
        if masters is True:
            masters = [p.detach().float() for p in self.params]
        self.masters = list(masters) if masters is not None else None
        if self.masters is not None and dtype != torch.bfloat16:
            raise ValueError("masters: only for bfloat16 params")

        def state(given, dtype, counts):
            if given is not None:
                return list(given)
            return [torch.zeros(n, dtype=torch.uint8, device=self._dev).view(dtype)
                    if dtype == torch.float8_e4m3fn else
                    torch.zeros(n, dtype=dtype, device=self._dev) for n in counts]
        kind = torch.float8_e4m3fn if state_bits == 8 else torch.float32
        self.exp_avg, self.exp_avg_sq = state(exp_avg, kind, sizes), state(exp_avg_sq, kind, sizes)
        self.exp_avg_scale = self.exp_avg_sq_scale = None
        scales = [-(-n // ADAMW_BLOCK) for n in sizes]
        if state_bits == 8:
            self.exp_avg_scale = state(exp_avg_scale, torch.float32, scales)
            self.exp_avg_sq_scale = state(exp_avg_sq_scale, torch.float32, scales)
        elif exp_avg_scale is not None or exp_avg_sq_scale is not None:
            raise ValueError("scales: only for 8-bit states")
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * len(sizes)
        self._table = (AdamWTensor * len(sizes))()
        self._memory = []                        # what the table's addresses point to
        self._fill("param", self.params, sizes, dtype)
        self._fill("master", self.masters, sizes, torch.float32)
        self._fill("exp_avg", self.exp_avg, sizes, kind)
        self._fill("exp_avg_sq", self.exp_avg_sq, sizes, kind)
        self._fill("exp_avg_scale", self.exp_avg_scale, scales, torch.float32)
        self._fill("exp_avg_sq_scale", self.exp_avg_sq_scale, scales, torch.float32)
        if len(decay) != len(sizes):
            raise ValueError(f"weight_decay: {len(decay)} values for {len(sizes)} tensors")
        for row, n, wd in zip(self._table, sizes, decay):
            row.n, row.weight_decay = n, wd
        self._config = AdamWConfig(_ACT[dtype], 0, int(self.masters is not None), state_bits, 1, 0.0,
                                   float(betas[0]), float(betas[1]), float(eps))
        self.grads = None
        if grads is not None:
            self.set_grads(grads)

    def _addresses(self, field, tensors, sizes, dtype):
        """The addresses of a list of tensors, every one of them checked."""
        if len(tensors) != len(sizes):
            raise ValueError(f"{field}: {len(tensors)} tensors for {len(sizes)} params")
        at = []
        for i, (t, n) in enumerate(zip(tensors, sizes)):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{field}[{i}]: expected a torch.Tensor")
            if t.numel() != n:
                raise ValueError(f"{field}[{i}]: {t.numel()} elements, expected {n}")
            _expect(f"{field}[{i}]", t, t.shape, dtype, self._dev)
            at.append(_ptr(t).value)
        return at

    def _fill(self, field, tensors, sizes, dtype):
        if tensors is None:
            return
        for row, at in zip(self._table, self._addresses(field, tensors, sizes, dtype)):
            setattr(row, field, at)
        self._memory += [t.detach() for t in tensors]

    def set_grads(self, grads):
        """Exchanges the gradients of the steps to come: all of them, or none where one is refused."""
        grads = list(grads)
        dtype = grads[0].dtype if grads and isinstance(grads[0], torch.Tensor) else None
        if dtype not in _ACT:
            raise ValueError(f"grads: dtype {dtype}, expected float32 or bfloat16")
        addresses = self._addresses("grad", grads, [p.numel() for p in self.params], dtype)
        for row, at in zip(self._table, addresses):
            row.grad = at
        self._config.grad_dtype = _ACT[dtype]
        self.grads = grads

    def scalars(self, step, lr):
        """What a step's `scalars` tensor has to hold for this step and learning rate."""
        c = self._config
        return [lr, 1.0 / (1.0 - c.beta1 ** step), 1.0 / (1.0 - c.beta2 ** step) ** 0.5]

    def step(self, step, lr, *, grad_scale=None, scalars=None, stream=None):
        """Step number `step` (from 1).  grad_scale: [1] float32 on the device, multiplies every
        gradient; not finite = the step is skipped.  scalars: [3] float32 on the device with the
        values of self.scalars(), used instead of step and lr (for a captured step)."""
        if self._dev.index != torch.cuda.current_device():
            raise ValueError(f"AdamW: tensors on {self._dev}, which is not the current device")
        self._config.step, self._config.lr = int(step), float(lr)
        _check(lib.r3_adamw_step(ctypes.byref(self._config), self._table, len(self.params),
                                 _arg("grad_scale", grad_scale, (1,), torch.float32, self._dev),
                                 _arg("scalars", scalars, (3,), torch.float32, self._dev),
                                 _stream(stream)))


def _block_norms(s, L, w_pre, w_post, gate, eps, residual_scale, branch_scale, dev, grads):
    """The r3_block_norms of a call, its vectors [L, d] checked, and (grads) their gradients."""
    if not isinstance(w_pre, torch.Tensor) or w_pre.dtype not in _ACT:
        raise ValueError("w_pre: expected a float32 or bfloat16 tensor")
    n = BlockNorms(w_dtype=_ACT[w_pre.dtype], eps=eps, residual_scale=residual_scale,
                   branch_scale=branch_scale)
    new = torch.empty if s.T else torch.zeros    # an empty batch's sums are written by nothing
    made = []
    for name, t, grad in (("w_pre", w_pre, "dw_pre"), ("w_post", w_post, "dw_post"), ("gate", gate, "dgate")):
        setattr(n, name, _arg(name, t, (L, s.d), w_pre.dtype, dev))
        g = new((L, s.d), dtype=torch.float32, device=dev) if grads and t is not None else None
        setattr(n, grad, None if g is None else g.data_ptr())
        made.append(g)
    return n, made


def _stack_inputs(s, L, w_router, idx, w_gate, w_up, w_down, dev):
    """The addresses of a stack's routers, records and expert weights, each of the type that the shape says
    and with all L layers."""
    router = torch.bfloat16 if s.router_w_dtype == R3_BF16 else torch.float32
    expert, act = L * s.E * s.F * s.d, _act_dtype(s)
    at = []
    for name, t, n, dtype in (("w_router", w_router, L * s.E * s.d, router),
                              ("idx", idx, L * s.T * s.K, _idx_dtype(s)), ("w_gate", w_gate, expert, act),
                              ("w_up", w_up, expert, act), ("w_down", w_down, expert, act)):
        if not isinstance(t, torch.Tensor):
            raise TypeError(f"{name}: expected a torch.Tensor")
        if t.numel() != n:
            raise ValueError(f"{name}: {t.numel()} elements, expected {n} ({L} layers)")
        at.append(_arg(name, t, t.shape, dtype, dev))
    return at


@_in_order
def normed_stack(s: Shape, L: int, x0, w_router, idx, w_gate, w_up, w_down, *, w_pre, w_post=None,
                 gate=None, eps=1e-6, residual_scale=1.0, branch_scale=1.0, x_out=None, ws=None,
                 dev_status=None, stream=None):
    """L replayed blocks with norms around them (vectors w_pre, w_post, gate [L, d]), forward:
    x_{l+1} = residual_scale x_l + branch_scale gate_l RMSNorm(y_l(RMSNorm(x_l) w_pre_l)) w_post_l.
    Returns x_L [T, d]."""
    dev = _device_of("x0", x0)
    n, _ = _block_norms(s, L, w_pre, w_post, gate, eps, residual_scale, branch_scale, dev, False)
    layers = _stack_inputs(s, L, w_router, idx, w_gate, w_up, w_down, dev)
    x0 = _arg("x0", x0, (s.T, s.d), _act_dtype(s), dev)
    if x_out is None:
        x_out = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    ws = _scratch(ws, lib.r3_normed_stack_workspace_bytes(ctypes.byref(s)), dev)
    _check(lib.r3_normed_stack(ctypes.byref(s), L, ctypes.byref(n), x0, *layers,
                               _arg("x_out", x_out, (s.T, s.d), _act_dtype(s), dev), _ptr(ws),
                               ws.numel(), _ptr(dev_status), _stream(stream)))
    return x_out


@_in_order
def normed_stack_train(s: Shape, L: int, x0, w_router, idx, w_gate, w_up, w_down, dy, *, w_pre,
                       w_post=None, gate=None, eps=1e-6, residual_scale=1.0, branch_scale=1.0,
                       expert_grads=False, optimiser=None, step=None, lr=None, grad_scale=None,
                       scalars=None, ws=None, dev_status=None, stream=None):
    """normed_stack forward and the exact backward chain of <dy, x_L>: (x_out, dlogits [L, T, E], dx0,
    dw_router [L, E, d], dw_pre, dw_post or None, dgate or None), and with expert_grads also (dw_gate,
    dw_up, dw_down).  With optimiser, an AdamW over [w_gate[0], w_up[0], w_down[0], w_gate[1], ..] without
    gradients of its own, every block's expert weights take step `step` with rate `lr` as soon as their
    gradients are there, and only one block's gradients exist at a time (block 0's are returned).  Without
    rows the gradients are zero and no step is taken; nor is one once dev_status holds an error, of this call
    (noticed without a dev_status too) or from before."""
    dev = _device_of("x0", x0)
    n, dnorms = _block_norms(s, L, w_pre, w_post, gate, eps, residual_scale, branch_scale, dev, True)
    layers = _stack_inputs(s, L, w_router, idx, w_gate, w_up, w_down, dev)
    x0, dy = (_arg(name, t, (s.T, s.d), _act_dtype(s), dev) for name, t in (("x0", x0), ("dy", dy)))
    f32 = dict(dtype=torch.float32, device=dev)
    x_out = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    dx0 = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    new = torch.empty if s.T else torch.zeros
    dlogits = torch.empty((L, s.T, s.E), **f32)
    dw_r = new((L, s.E, s.d), **f32)
    dws, config, table = (None, None, None), None, None
    if optimiser is not None:
        if len(optimiser.params) != 3 * L:
            raise ValueError(f"optimiser: {len(optimiser.params)} tensors, expected {3 * L}")
        config = AdamWConfig.from_buffer_copy(optimiser._config)
        config.grad_dtype, config.step, config.lr = R3_F32, int(step), float(lr)
        table = optimiser._table
    if expert_grads or optimiser is not None:
        lead = () if optimiser is not None else (L,)
        dws = (new(lead + (s.E, s.F, s.d), **f32), new(lead + (s.E, s.F, s.d), **f32),
               new(lead + (s.E, s.d, s.F), **f32))
    ws = _scratch(ws, lib.r3_normed_stack_train_workspace_bytes(ctypes.byref(s), L), dev)
    _check(lib.r3_normed_stack_train(
        ctypes.byref(s), L, ctypes.byref(n), x0, *layers, dy, _ptr(x_out), _ptr(dlogits), _ptr(dx0), _ptr(dw_r),
        _ptr(dws[0]), _ptr(dws[1]), _ptr(dws[2]), None if config is None else ctypes.addressof(config),
        None if table is None else ctypes.addressof(table),
        _arg("grad_scale", grad_scale, (1,), torch.float32, dev),
        _arg("scalars", scalars, (3,), torch.float32, dev), _ptr(ws), ws.numel(), _ptr(dev_status),
        _stream(stream)))
    out = (x_out, dlogits, dx0, dw_r, *dnorms)
    return out + dws if dws[0] is not None else out


def _rows(name: str, t):
    """Pointer and row stride of a [T, V] tensor whose rows may lie apart but are dense."""
    if t.dim() != 2:
        raise ValueError(f"{name}: expected [T, V]")
    (rows, width), (ld, hop) = t.shape, t.stride()
    if width > 1 and hop != 1:
        raise ValueError(f"{name}: expected [T, V] with adjacent columns")
    if rows <= 1:
        ld = width
    elif ld < width:
        raise ValueError(f"{name}: rows overlap")
    return t.data_ptr(), ld


def _logits_shape(logits, token_ids, temperature):
    """The r3_logits of a call and the addresses of the logits and the ids (None without)."""
    dev = _device_of("logits", logits)
    dtype = _ACT.get(logits.dtype)
    if dtype is None:
        raise ValueError(f"logits: dtype {logits.dtype}, expected float32 or bfloat16")
    ptr, ld = _rows("logits", logits)
    T, V = logits.shape
    ids, id_bytes = None, 4
    if token_ids is not None:
        wide = token_ids.dtype != torch.int32
        id_bytes = 8 if wide else 4
        ids = _arg("token_ids", token_ids, (T,), torch.int64 if wide else torch.int32, dev)
    return Logits(T, V, ld, dtype, id_bytes, temperature), ptr, ids, dev


@_in_order
def token_logprobs(logits, token_ids=None, *, temperature=1.0, n_top=0, want_entropy=False,
                   want_stats=False, dev_status=None, stream=None):
    """Log probabilities of token_ids [T] (int32 or int64) under logits [T, V] (float32 or bfloat16;
    rows may lie apart).  Returns (logp [T] or None without token_ids, entropy [T] or None,
    stats [T, 2] or None, top_ids [T, n_top] int32 or None, top_logp [T, n_top] or None).  A row
    with a negative token id is skipped: zeros, top_ids -1."""
    s, ptr, ids, dev = _logits_shape(logits, token_ids, temperature)
    new, f32, T = torch.empty_strided, torch.float32, s.T    # the cheapest of torch's allocating calls
    logp = entropy = stats = top_ids = top_logp = None
    at = [None] * 5                              # the outputs' addresses
    if ids is not None:
        logp = new((T,), (1,), dtype=f32, device=dev)
        at[0] = logp.data_ptr()
    if want_entropy:
        entropy = new((T,), (1,), dtype=f32, device=dev)
        at[1] = entropy.data_ptr()
    if want_stats:
        stats = new((T, 2), (2, 1), dtype=f32, device=dev)
        at[2] = stats.data_ptr()
    if n_top > 0:
        top_ids = new((T, n_top), (n_top, 1), dtype=torch.int32, device=dev)
        top_logp = new((T, n_top), (n_top, 1), dtype=f32, device=dev)
        at[3], at[4] = top_ids.data_ptr(), top_logp.data_ptr()
    _check(lib.r3_token_logprobs(ctypes.byref(s), ptr, ids, at[0], at[1], at[2], n_top, at[3], at[4],
                                 None if dev_status is None else _ptr(dev_status), _stream(stream)))
    return logp, entropy, stats, top_ids, top_logp


@_in_order
def token_logprobs_bwd(logits, token_ids, stats, dlogp, *, entropy=None, dentropy=None,
                       temperature=1.0, dlogits=None, dev_status=None, stream=None):
    """Gradient to the logits from dlogp [T] (or None) and, with the forward's entropy [T], from
    dentropy [T].  stats [T, 2] and temperature as in the forward.  dlogits may be given (the logits
    themselves, for a gradient in place)."""
    s, ptr, ids, dev = _logits_shape(logits, token_ids, temperature)
    if dlogits is None:
        dlogits = torch.empty_strided((s.T, s.V), (s.V, 1), dtype=logits.dtype, device=dev)
    else:
        _expect("dlogits", dlogits, (s.T, s.V), logits.dtype, dev)
    out, ld_out = _rows("dlogits", dlogits)
    stats = _arg("stats", stats, (s.T, 2), torch.float32, dev)
    entropy, dlogp, dentropy = (_arg(name, t, (s.T,), torch.float32, dev) for name, t in
                                (("entropy", entropy), ("dlogp", dlogp), ("dentropy", dentropy)))
    _check(lib.r3_token_logprobs_bwd(ctypes.byref(s), ptr, ids, stats, entropy, dlogp, dentropy, out,
                                     ld_out, _ptr(dev_status), _stream(stream)))
    return dlogits


@_in_order
def prob_discrepancy(p_train, p_infer, taus, *, kl=None, counts=None, ws=None, stream=None):
    """k3 KL estimate (Eq. kl) and extreme-token counts (Eq. etdf) of two float32 probability
    arrays.  `taus`: a list or a float32 device tensor.  Returns (kl [1] float64, counts [n_tau]
    int64); F(tau) = counts / n."""
    dev = _dev(p_train)
    n = p_train.numel()
    if not (isinstance(taus, torch.Tensor) and taus.is_cuda and taus.dtype == torch.float32):
        taus = torch.as_tensor(taus, dtype=torch.float32, device=dev).contiguous()
    if kl is None:
        kl = torch.empty(1, dtype=torch.float64, device=dev)
    if counts is None:
        counts = torch.empty(taus.numel(), dtype=torch.int64, device=dev)
    if ws is None:
        ws = workspace(lib.r3_prob_discrepancy_workspace_bytes(n), dev)
    _check(lib.r3_prob_discrepancy(_ptr(p_train), _ptr(p_infer), n, _ptr(taus), taus.numel(),
                                   _ptr(kl), _ptr(counts), _ptr(ws), ws.numel(), _stream(stream)))
    return kl, counts


@_in_order
def record_diff(s: Shape, L: int, rec_a, rec_b, *, want_diff=True, stream=None):
    """Differing expert choices between two records [L,T,K].  Returns (diff [L,T] uint8 or None,
    token_choices [T], token_routers [T], hist [K+1] int64)."""
    dev = _dev(rec_a)
    diff = torch.empty((L, s.T), dtype=torch.uint8, device=dev) if want_diff else None
    choices = torch.empty(s.T, dtype=torch.int32, device=dev)
    routers = torch.empty(s.T, dtype=torch.int32, device=dev)
    hist = torch.empty(s.K + 1, dtype=torch.int64, device=dev)
    _check(lib.r3_record_diff(ctypes.byref(s), L, _ptr(rec_a), _ptr(rec_b), _ptr(diff),
                              _ptr(choices), _ptr(routers), _ptr(hist), _stream(stream)))
    return diff, choices, routers, hist


@_in_order
def sequence_diff(token_routers, cu_seqlens, *, stream=None):
    """Per-sequence sums of token_routers over [cu_seqlens[s], cu_seqlens[s+1])."""
    S = cu_seqlens.numel() - 1
    out = torch.empty(S, dtype=torch.int64, device=_dev(token_routers))
    _check(lib.r3_sequence_diff(_ptr(token_routers), _ptr(cu_seqlens), S, _ptr(out),
                                _stream(stream)))
    return out


# ---------------------------------------------------------------------------------------------
def record_page_bytes(s: Shape, L: int, page_tokens: int) -> int:
    return lib.r3_record_page_bytes(ctypes.byref(s), L, page_tokens)


def record_append(s: Shape, L: int, page_tokens: int, pages, block_table, seq_pos0, cu_new,
                  rec_new, *, dev_status=None, stream=None):
    """Writes rec_new [L, N, K] (N new tokens, packed by cu_new) into the pages of their sequences."""
    n_pages = pages.numel() // record_page_bytes(s, L, page_tokens)
    B, max_pages = block_table.shape
    _check(lib.r3_record_append(ctypes.byref(s), L, page_tokens, n_pages, _ptr(pages),
                                _ptr(block_table), max_pages, _ptr(seq_pos0), _ptr(cu_new), B,
                                _ptr(rec_new), rec_new.shape[1], _ptr(dev_status), _stream(stream)))


@_in_order
def record_gather(s: Shape, L: int, page_tokens: int, pages, block_table, cu_seqlens, T: int, *,
                  out=None, dev_status=None, stream=None):
    """The packed record [L, T, K] of a variable-length batch, assembled from the pages."""
    n_pages = pages.numel() // record_page_bytes(s, L, page_tokens)
    B, max_pages = block_table.shape
    if out is None:
        out = torch.empty((L, T, s.K), dtype=_idx_dtype(s), device=_dev(pages))
    _check(lib.r3_record_gather(ctypes.byref(s), L, page_tokens, n_pages, _ptr(pages),
                                _ptr(block_table), max_pages, _ptr(cu_seqlens), B, _ptr(out), T,
                                _ptr(dev_status), _stream(stream)))
    return out


class PagePool:
    """Host-side page bookkeeping of the record store (r3_pagepool_*): lists in, lists out."""

    def __init__(self, n_pages: int, page_tokens: int):
        self.page_tokens = page_tokens
        self._h = lib.r3_pagepool_create(n_pages, page_tokens)
        if not self._h:
            raise ValueError("r3_pagepool_create failed")

    def close(self):
        if self._h:
            lib.r3_pagepool_destroy(self._h)
            self._h = None

    __del__ = close

    @staticmethod
    def _arr(v):
        return (ctypes.c_int32 * max(len(v), 1))(*v)

    def free_pages(self) -> int:
        return lib.r3_pagepool_free_pages(self._h)

    def match(self, token_ids) -> list:
        cap = len(token_ids) // self.page_tokens
        out = (ctypes.c_int32 * max(cap, 1))()
        n = lib.r3_pagepool_match(self._h, self._arr(token_ids), len(token_ids), out, cap)
        return list(out[:n])

    def alloc(self, n: int) -> list:
        out = (ctypes.c_int32 * max(n, 1))()
        _check(lib.r3_pagepool_alloc(self._h, n, out))
        return list(out[:n])

    def publish(self, token_ids, table) -> None:
        _check(lib.r3_pagepool_publish(self._h, self._arr(token_ids), len(token_ids),
                                       self._arr(table), len(table)))

    def release(self, table) -> None:
        _check(lib.r3_pagepool_release(self._h, self._arr(table), len(table)))


@_in_order
def grouped_swiglu_train(s: Shape, xp, offsets, w_gate, w_up, w_down, *, ws=None, dev_status=None,
                         stream=None):
    """Grouped experts that also return the pre-activations: (o [R,d], pre_gate, pre_up [R,F])."""
    dev = _dev(xp)
    R = s.T * s.K
    o = torch.empty((R, s.d), dtype=_act_dtype(s), device=dev)
    pre_gate = torch.empty((R, s.F), dtype=_act_dtype(s), device=dev)
    pre_up = torch.empty((R, s.F), dtype=_act_dtype(s), device=dev)
    if ws is None:
        ws = workspace(lib.r3_grouped_swiglu_workspace_bytes(ctypes.byref(s)), dev)
    _check(lib.r3_grouped_swiglu_train(ctypes.byref(s), _ptr(xp), _ptr(offsets), _ptr(w_gate),
                                       _ptr(w_up), _ptr(w_down), _ptr(o), _ptr(pre_gate),
                                       _ptr(pre_up), _ptr(ws), ws.numel(), _ptr(dev_status),
                                       _stream(stream)))
    return o, pre_gate, pre_up


@_in_order
def scale_rows(s: Shape, dy, gates, row_of_slot, dout=None, *, stream=None):
    """dout[row_of_slot[t,j]] = gates[t,j] * dy[t]."""
    if dout is None:
        dout = torch.empty((s.T * s.K, s.d), dtype=_act_dtype(s), device=_dev(dy))
    _check(lib.r3_scale_rows(ctypes.byref(s), _ptr(dy), _ptr(gates), _ptr(row_of_slot),
                             _ptr(dout), _stream(stream)))
    return dout


@_in_order
def input_grad_finish(s: Shape, dxp, row_of_slot, slot_of_row, offsets, dlogits, idx, x, w_router,
                      *, dx_residual=None, stream=None):
    """(dx [T,d], dw_router [E,d] float32) from the expert input gradient and dlogits."""
    dev = _dev(dxp)
    dx = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    dw_r = torch.empty((s.E, s.d), dtype=torch.float32, device=dev)
    _check(lib.r3_input_grad_finish(ctypes.byref(s), _ptr(dxp), _ptr(row_of_slot),
                                    _ptr(slot_of_row), _ptr(offsets), _ptr(dlogits), _ptr(idx),
                                    _ptr(x), _ptr(w_router), _ptr(dx_residual), _ptr(dx),
                                    _ptr(dw_r), _stream(stream)))
    return dx, dw_r


@_in_order
def grouped_swiglu_bwd(s: Shape, xp, dout, pre_gate, pre_up, offsets, w_gate, w_up, w_down, *,
                       ws=None, dev_status=None, stream=None):
    """Backward of the grouped experts: (dxp [R,d], dw_gate, dw_up [E,F,d], dw_down [E,d,F])."""
    dev = _dev(dout)
    dxp = torch.empty((s.T * s.K, s.d), dtype=_act_dtype(s), device=dev)
    dw_gate = torch.empty((s.E, s.F, s.d), dtype=torch.float32, device=dev)
    dw_up = torch.empty((s.E, s.F, s.d), dtype=torch.float32, device=dev)
    dw_down = torch.empty((s.E, s.d, s.F), dtype=torch.float32, device=dev)
    if ws is None:
        ws = workspace(lib.r3_grouped_swiglu_bwd_workspace_bytes(ctypes.byref(s)), dev)
    _check(lib.r3_grouped_swiglu_bwd(ctypes.byref(s), _ptr(xp), _ptr(dout), _ptr(pre_gate),
                                     _ptr(pre_up), _ptr(offsets), _ptr(w_gate), _ptr(w_up),
                                     _ptr(w_down), _ptr(dxp), _ptr(dw_gate), _ptr(dw_up),
                                     _ptr(dw_down), _ptr(ws), ws.numel(), _ptr(dev_status),
                                     _stream(stream)))
    return dxp, dw_gate, dw_up, dw_down


@_in_order
def replay_layer_train(s: Shape, x, w_router, idx, w_gate, w_up, w_down, dy, *, ws=None,
                       dev_status=None, stream=None, expert_grads=False, dw_experts=None):
    """Forward and backward of one replayed layer: (y, dlogits, dx, dw_router), and with
    expert_grads also (dw_gate, dw_up, dw_down) appended (float32; `dw_experts` may supply the
    three output tensors)."""
    dev = _dev(x)
    y = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    dlogits = torch.empty((s.T, s.E), dtype=torch.float32, device=dev)
    dx = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    dw_r = torch.empty((s.E, s.d), dtype=torch.float32, device=dev)
    if ws is None:
        ws = workspace(lib.r3_replay_layer_train_workspace_bytes(ctypes.byref(s)), dev)
    dws = (None, None, None)
    if expert_grads:
        dws = dw_experts or (
            torch.empty((s.E, s.F, s.d), dtype=torch.float32, device=dev),
            torch.empty((s.E, s.F, s.d), dtype=torch.float32, device=dev),
            torch.empty((s.E, s.d, s.F), dtype=torch.float32, device=dev))
    _check(lib.r3_replay_layer_train(ctypes.byref(s), _ptr(x), _ptr(w_router), _ptr(idx),
                                     _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(dy), _ptr(y),
                                     _ptr(dlogits), _ptr(dx), _ptr(dw_r), _ptr(dws[0]),
                                     _ptr(dws[1]), _ptr(dws[2]), _ptr(ws), ws.numel(),
                                     _ptr(dev_status), _stream(stream)))
    if expert_grads:
        return (y, dlogits, dx, dw_r) + tuple(dws)
    return y, dlogits, dx, dw_r


@_in_order
def replay_stack_train(s: Shape, L, x0, w_router, idx, w_gate, w_up, w_down, dy, *, ws=None,
                       dev_status=None, stream=None, expert_grads=False):
    """L residual blocks forward, then the exact backward chain:
    (x_out, dlogits [L,T,E], dx0, dw_router [L,E,d]) (+ dw_gate, dw_up, dw_down)."""
    dev = _dev(x0)
    x_out = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    dx0 = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    dlogits = torch.empty((L, s.T, s.E), dtype=torch.float32, device=dev)
    dw_r = torch.empty((L, s.E, s.d), dtype=torch.float32, device=dev)
    dws = (None, None, None)
    if expert_grads:
        dws = (torch.empty((L, s.E, s.F, s.d), dtype=torch.float32, device=dev),
               torch.empty((L, s.E, s.F, s.d), dtype=torch.float32, device=dev),
               torch.empty((L, s.E, s.d, s.F), dtype=torch.float32, device=dev))
    if ws is None:
        ws = workspace(lib.r3_replay_stack_train_workspace_bytes(ctypes.byref(s), L), dev)
    _check(lib.r3_replay_stack_train(ctypes.byref(s), L, _ptr(x0), _ptr(w_router), _ptr(idx),
                                     _ptr(w_gate), _ptr(w_up), _ptr(w_down), _ptr(dy),
                                     _ptr(x_out), _ptr(dlogits), _ptr(dx0), _ptr(dw_r),
                                     _ptr(dws[0]), _ptr(dws[1]), _ptr(dws[2]), _ptr(ws),
                                     ws.numel(), _ptr(dev_status), _stream(stream)))
    if expert_grads:
        return (x_out, dlogits, dx0, dw_r) + dws
    return x_out, dlogits, dx0, dw_r


@_in_order
def ep_regroup_map(recv_counts, rows: int, *, dev_status=None, stream=None):
    """recv_counts [n_src, e_local] int32 (device) -> (perm [rows] int32, offsets [e_local+1])."""
    n_src, e_local = recv_counts.shape
    dev = _dev(recv_counts)
    perm = torch.empty(max(rows, 1), dtype=torch.int32, device=dev)[:rows]
    offsets = torch.empty(e_local + 1, dtype=torch.int32, device=dev)
    _check(lib.r3_ep_regroup_map(_ptr(recv_counts), n_src, e_local, rows,
                                 _ptr(perm) if rows else None, _ptr(offsets), _ptr(dev_status),
                                 _stream(stream)))
    return perm, offsets


def _peer_array(addresses):
    return (ctypes.c_uint64 * len(addresses))(*[int(a) for a in addresses])


@_in_order
def ep_dest_table(counts_all, rank: int, *, stream=None):
    """counts_all [n_ranks, E] int32 (device) -> (dst_base [E], offsets_local [E/n_ranks + 1])."""
    n, E = counts_all.shape
    dev = _dev(counts_all)
    dst_base = torch.empty(E, dtype=torch.int32, device=dev)
    offsets_local = torch.empty(E // n + 1, dtype=torch.int32, device=dev)
    _check(lib.r3_ep_dest_table(_ptr(counts_all), n, E, rank, _ptr(dst_base), _ptr(offsets_local),
                                _stream(stream)))
    return dst_base, offsets_local


def ep_dispatch_rows(s: Shape, n_ranks: int, x, idx, row_of_slot, my_offsets, dst_base,
                     peer_addresses, capacity_rows: int, *, dev_status=None, stream=None):
    """x[t] straight into the owners' receive buffers (peer_addresses: their base addresses,
    capacity_rows rows each; a row beyond the capacity is dropped and flagged)."""
    arr = _peer_array(peer_addresses)
    _check(lib.r3_ep_dispatch_rows(ctypes.byref(s), n_ranks, _ptr(x), _ptr(idx), _ptr(row_of_slot),
                                   _ptr(my_offsets), _ptr(dst_base), arr, int(capacity_rows),
                                   _ptr(dev_status), _stream(stream)))


@_in_order
def ep_slot_rows(s: Shape, n_ranks: int, idx, row_of_slot, my_offsets, dst_base, peer_addresses,
                 capacity_rows: int, *, dev_status=None, stream=None):
    """[T, K] addresses of the pairs' expert-output rows in the owners' output buffers."""
    row_ptr = torch.empty((s.T, s.K), dtype=torch.int64, device=_dev(idx))
    arr = _peer_array(peer_addresses)
    _check(lib.r3_ep_slot_rows(ctypes.byref(s), n_ranks, _ptr(idx), _ptr(row_of_slot),
                               _ptr(my_offsets), _ptr(dst_base), arr, int(capacity_rows),
                               _ptr(row_ptr), _ptr(dev_status), _stream(stream)))
    return row_ptr


@_in_order
def replay_finish_rows(s: Shape, logits, idx, row_ptr, dy, *, residual=None, dev_status=None,
                       stream=None):
    """r3_replay_finish with the expert-output rows given by address.  (y, gates, dlogits)."""
    dev = _dev(idx)
    y = torch.empty((s.T, s.d), dtype=_act_dtype(s), device=dev)
    gates = torch.empty((s.T, s.K), dtype=torch.float32, device=dev)
    dlogits = torch.empty((s.T, s.E), dtype=torch.float32, device=dev)
    _check(lib.r3_replay_finish_rows(ctypes.byref(s), _ptr(logits), _ptr(idx), _ptr(row_ptr),
                                     _ptr(dy), _ptr(residual), _ptr(y), _ptr(gates), _ptr(dlogits),
                                     _ptr(dev_status), _stream(stream)))
    return y, gates, dlogits


@_in_order
def ep_move_rows(src, perm, *, inverse=False, stream=None):
    """Rows of `src` [rows, width] reordered by `perm` (see r3_ep_move_rows)."""
    dst = torch.empty_like(src)
    rows = src.shape[0]
    if rows:
        _check(lib.r3_ep_move_rows(_ptr(src), _ptr(dst), _ptr(perm), rows,
                                   src.shape[1] * src.element_size(), 1 if inverse else 0,
                                   _stream(stream)))
    return dst


@_in_order
def grouped_swiglu_bwd_input(s: Shape, dout, pre_gate, pre_up, offsets, w_gate, w_up, w_down,
                             dxp=None, *, ws=None, dev_status=None, stream=None):
    """Input gradient of the grouped SwiGLU experts: dout [R,d] -> dxp [R,d] (bf16)."""
    dev = _dev(dout)
    if dxp is None:
        dxp = torch.empty((s.T * s.K, s.d), dtype=_act_dtype(s), device=dev)
    if ws is None:
        ws = workspace(lib.r3_grouped_swiglu_bwd_workspace_bytes(ctypes.byref(s)), dev)
    _check(lib.r3_grouped_swiglu_bwd_input(ctypes.byref(s), _ptr(dout), _ptr(pre_gate),
                                           _ptr(pre_up), _ptr(offsets), _ptr(w_gate), _ptr(w_up),
                                           _ptr(w_down), _ptr(dxp), _ptr(ws), ws.numel(),
                                           _ptr(dev_status), _stream(stream)))
    return dxp


@_in_order
def selftest_bounded_wait(limit_clocks: int, *, dev_status=None, device="cuda", stream=None):
    """Makes the library's bounded barrier wait run out on purpose (a barrier nothing signals).
    Returns out [4] int32: (wait result, abort flag, clocks waited, result of a second wait)."""
    out = torch.full((4,), -1, dtype=torch.int32, device=device)
    _check(lib.r3_selftest_bounded_wait(int(limit_clocks), _ptr(dev_status), _ptr(out),
                                        _stream(stream)))
    return out
