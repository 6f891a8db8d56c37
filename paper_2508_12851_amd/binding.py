"""Thin ctypes binding of libprism's C ABI (include/prism.h).

Argument marshalling only: every step of the layer runs in the HIP kernels of
libprism.so.  PyTorch is used for device memory and streams.  There is no CPU
fallback: if the library is missing, or a call fails, an exception is raised.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libprism.so")

PRISM_F32, PRISM_BF16 = 0, 1
SYMBOLS = ("prism_status_string", "prism_workspace_bytes", "prism_route", "prism_dispatch",
           "prism_expert_ffn", "prism_combine", "prism_moe_layer", "prism_moe_layer_traced",
           "prism_ceiling_mfma_bf16", "prism_ceiling_hbm_read", "prism_pack_remote",
           "prism_combine_remote", "prism_debug_check_weights", "prism_pack_weights",
           "prism_layer_permutation", "prism_moe_layer_static", "prism_ceiling_hbm_read_pattern",
           "prism_clear_rows", "prism_balance_workspace_bytes", "prism_balance_loss", "prism_route_backward",
           "prism_i8_bytes", "prism_quantize_i8", "prism_pack_i8", "prism_matmul_i8_workspace_bytes", "prism_matmul_i8")
STAGES = ("route", "dispatch", "ffn_up", "ffn_down", "combine")
GATE_MODES = {"renormalized": 0, "softmax_all": 1}
WEIGHT_LAYOUTS = {"row_major": 0, "tiled": 1, "int8": 2}


class PrismError(RuntimeError):
    pass


class LayerDesc(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("ffn", ctypes.c_int32), ("n_experts", ctypes.c_int32),
                ("top_k", ctypes.c_int32), ("n_shared", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("bias_group_tokens", ctypes.c_int32), ("gate_mode", ctypes.c_int32),
                ("weight_layout", ctypes.c_int32)]


class ExpertWeights(ctypes.Structure):
    _fields_ = [("w_gate", ctypes.c_void_p), ("w_up", ctypes.c_void_p), ("w_down", ctypes.c_void_p),
                ("shared_w_gate", ctypes.c_void_p), ("shared_w_up", ctypes.c_void_p),
                ("shared_w_down", ctypes.c_void_p)]


_lib = None


def load_library(build_if_missing: bool = True) -> ctypes.CDLL:
    """Load libprism.so (building it in-tree first if it does not exist)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        if not build_if_missing:
            raise PrismError(f"{LIB_PATH} is not built; run python -m paper_2508_12851_amd.build")
        from . import build as _build
        _build.build_library(verbose=False)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    dp = ctypes.POINTER(LayerDesc)
    wp = ctypes.POINTER(ExpertWeights)
    lib.prism_status_string.restype = ctypes.c_char_p
    lib.prism_status_string.argtypes = [ctypes.c_int]
    lib.prism_workspace_bytes.argtypes = [dp, i32, ctypes.POINTER(sz)]
    lib.prism_route.argtypes = [dp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.prism_balance_workspace_bytes.argtypes = [dp, ctypes.POINTER(sz)]
    lib.prism_balance_loss.argtypes = [dp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.prism_route_backward.argtypes = [dp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp]
    i64 = ctypes.c_int64
    lib.prism_i8_bytes.argtypes = [i32, i32, ctypes.POINTER(sz)]
    lib.prism_quantize_i8.argtypes = [vp, i32, i64, i32, i32, vp, vp]
    lib.prism_pack_i8.argtypes = [vp, i64, vp, i32, i32, vp, vp]
    lib.prism_matmul_i8_workspace_bytes.argtypes = [i32, i32, i32, ctypes.POINTER(sz)]
    lib.prism_matmul_i8.argtypes = [vp, vp, i32, i32, i32, vp, i64, i32, vp, sz, vp]
    lib.prism_dispatch.argtypes = [dp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.prism_expert_ffn.argtypes = [dp, vp, wp, vp, vp, i32, vp, vp, sz, vp]
    lib.prism_combine.argtypes = [dp, vp, vp, vp, vp, i32, vp, vp, sz, vp]
    lib.prism_moe_layer.argtypes = [dp, vp, vp, vp, wp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                    vp, sz, vp]
    lib.prism_moe_layer_traced.argtypes = lib.prism_moe_layer.argtypes + [vp]
    lib.prism_moe_layer_static.argtypes = lib.prism_moe_layer.argtypes[:16] + [vp]
    lib.prism_pack_remote.argtypes = [dp, vp, vp, vp, i32, vp, vp]
    lib.prism_combine_remote.argtypes = [dp, vp, vp, vp, vp, i32, vp, vp, sz, vp]
    lib.prism_clear_rows.argtypes = [dp, vp, i32, vp, vp]
    lib.prism_pack_weights.argtypes = [vp, i32, i32, vp, vp]
    lib.prism_layer_permutation.argtypes = [dp, i32, vp, sz, vp, vp, vp, vp]
    lib.prism_debug_check_weights.argtypes = [dp, wp, vp, ctypes.POINTER(i32)]
    lib.prism_ceiling_mfma_bf16.argtypes = [vp, vp, i32, i32, ctypes.POINTER(ctypes.c_double), vp]
    lib.prism_ceiling_hbm_read.argtypes = [vp, sz, vp, i32, vp]
    lib.prism_ceiling_hbm_read_pattern.argtypes = [vp, sz, vp, i32, i32, sz, i32, ctypes.POINTER(sz), vp]
    for name in SYMBOLS:
        # without argtypes ctypes would pass a device address as a 32-bit int
        if getattr(lib, name).argtypes is None:
            raise PrismError(f"binding bug: no argument types declared for {name}")
    for name in SYMBOLS[1:]:
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def _check(code: int, what: str) -> None:
    if code != 0:
        msg = load_library().prism_status_string(code).decode()
        raise PrismError(f"{what}: {msg} (status {code})")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise PrismError("libprism takes contiguous device tensors")
    return t.data_ptr()


def _stream(stream: Optional[torch.cuda.Stream]) -> Optional[int]:
    # (the stream object of a device's current stream takes 2.5 us to make)
    return (torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) if stream is None else stream.cuda_stream) or None


def _stream_on(dev: int, stream: Optional[torch.cuda.Stream]) -> Optional[int]:
    """The stream of a call whose tensors are on device `dev`, the current one."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev) or None
    if stream.device_index != dev:
        raise PrismError(f"stream is on device {stream.device_index}, the call's tensors on {dev}")
    return stream.cuda_stream or None


_HERE = contextlib.nullcontext()


def _memory_of(stream: Optional[torch.cuda.Stream]):
    """Context in which the outputs of a call on `stream` are made (and filled): of that stream's memory.  What the current stream has
    freed, it may still have to read."""
    return _HERE if stream is None else torch.cuda.stream(stream)


def _new_on(stream: Optional[torch.cuda.Stream], like: torch.Tensor):
    """like.new_empty in that context."""
    if stream is None:
        return like.new_empty

    def new(shape, dtype=None):
        with torch.cuda.stream(stream):
            return like.new_empty(shape, dtype=dtype)
    return new


def make_desc(hidden: int, ffn: int, n_experts: int, top_k: int, n_shared: int = 0,
              dtype: str = "bf16", bias_group_tokens: int = 0,
              gate_mode: str = "renormalized", weight_layout: str = "row_major") -> LayerDesc:
    return LayerDesc(hidden, ffn, n_experts, top_k, n_shared,
                     PRISM_F32 if dtype == "f32" else PRISM_BF16, bias_group_tokens,
                     GATE_MODES[gate_mode], WEIGHT_LAYOUTS[weight_layout])


def torch_dtype(desc: LayerDesc) -> torch.dtype:
    return torch.float32 if desc.dtype == PRISM_F32 else torch.bfloat16


def _sizes_of(triples: Sequence) -> List[tuple]:
    """What is known of the gate, up and down matrices of some experts, for _check_sizes: the fewest bytes of one, the sizes of their
    elements, the (rows, cols) of those that are 8-bit matrices.  None for an expert that is not there."""
    out = []
    for i in range(3):
        ws = [t[i] for t in triples if t is not None]
        data = [w.data if isinstance(w, I8Matrix) else w for w in ws]
        out.append((min((d.numel() * d.element_size() for d in data), default=None), {d.element_size() for d in data},
                    {(w.rows, w.cols) for w in ws if isinstance(w, I8Matrix)}))
    return out


def _check_sizes(sizes: List[tuple], desc: LayerDesc) -> None:
    """Refuses matrices that the layer's calls would read beyond their end, or whose bytes are something else."""
    H, F, i8 = desc.hidden, desc.ffn, desc.weight_layout == WEIGHT_LAYOUTS["int8"]
    for (fewest, elements, shapes), (rows, cols), what in zip(sizes, ((F, H), (F, H), (H, F)), ("w_gate", "w_up", "w_down")):
        if fewest is None:
            continue
        if i8 and elements != {1}:
            raise PrismError(f"{what} has elements of {max(elements)} bytes in a layer with 8-bit weights")
        if shapes and not (i8 and shapes == {(rows, cols)}):
            raise PrismError(f"{what} has 8-bit matrices of {sorted(shapes)} in a layer that takes {'' if i8 else 'others, '}{rows} x {cols}")
        need = _i8_bytes(rows, cols) if i8 else rows * cols * (4 if desc.dtype == PRISM_F32 else 2)
        if fewest < need:
            raise PrismError(f"{what} has {fewest} bytes, {rows} x {cols} of this layer takes {need}")


class WeightTable:
    """Device arrays of device pointers to the expert weight matrices.

    experts[e] is (w_gate[F,H], w_up[F,H], w_down[H,F]) or None for an expert
    that is not hosted here; shared is a list of S such triples.  A matrix is a
    tensor or an I8Matrix.  They are kept alive by this object, and the calls
    refuse a table whose matrices are too small for the layer.
    """

    def __init__(self, experts: Sequence, shared: Sequence = (), device="cuda"):
        self.keep = (list(experts), list(shared))

        def table(items, i):
            ptrs = [0 if it is None else _ptr(it[i].data if isinstance(it[i], I8Matrix) else it[i]) for it in items]
            if not ptrs:
                return None
            return torch.tensor(ptrs, dtype=torch.int64, device=device)

        self.tables = [table(experts, i) for i in range(3)] + [table(shared, i) for i in range(3)]
        self.struct = ExpertWeights(*[None if t is None else t.data_ptr() for t in self.tables])
        self._sizes = _sizes_of(self.keep[0] + self.keep[1])
        self._fits = None           # (hidden, ffn, dtype, layout) that the matrices were last found large enough for

    def admit(self, e: int, triple: Sequence) -> None:
        """Keeps the matrices of routed expert e from now on; whoever calls this writes their addresses into the tables."""
        self.keep[0][e] = triple
        self._sizes = self._fits = None

    def struct_for(self, desc: LayerDesc):
        """The struct as the calls of this layer take it."""
        layer = (desc.hidden, desc.ffn, desc.dtype, desc.weight_layout)
        if self._fits != layer:
            if self._sizes is None:
                self._sizes = _sizes_of(self.keep[0] + self.keep[1])
            _check_sizes(self._sizes, desc)
            self._fits = layer
        return ctypes.byref(self.struct)


def workspace_bytes(desc: LayerDesc, max_tokens: int) -> int:
    n = ctypes.c_size_t(0)
    _check(load_library().prism_workspace_bytes(ctypes.byref(desc), max_tokens, ctypes.byref(n)),
           "prism_workspace_bytes")
    return n.value


def alloc_workspace(desc: LayerDesc, max_tokens: int, device="cuda") -> torch.Tensor:
    return torch.empty(workspace_bytes(desc, max_tokens), dtype=torch.uint8, device=device)


@dataclass
class RouteOut:
    logits: Optional[torch.Tensor]
    topk_idx: torch.Tensor
    topk_gate: torch.Tensor
    counts: torch.Tensor


def prism_route(desc: LayerDesc, x, w_router, router_bias, want_logits=True, counts_accum=None,
                stream=None) -> RouteOut:
    T, E, k = x.shape[0], desc.n_experts, desc.top_k
    dev = x.device
    with _memory_of(stream):
        logits = torch.empty((T, E), dtype=torch.float32, device=dev) if want_logits else None
        idx = torch.empty((T, k), dtype=torch.int32, device=dev)
        gate = torch.empty((T, k), dtype=torch.float32, device=dev)
        counts = torch.empty((E,), dtype=torch.int32, device=dev)
    _check(load_library().prism_route(ctypes.byref(desc), _ptr(x), _ptr(w_router), _ptr(router_bias),
                                      T, _ptr(logits), _ptr(idx), _ptr(gate), _ptr(counts),
                                      _ptr(counts_accum), _stream(stream)), "prism_route")
    return RouteOut(logits, idx, gate, counts)


def alloc_balance_workspace(desc: LayerDesc, device="cuda") -> torch.Tensor:
    n = ctypes.c_size_t(0)
    _check(load_library().prism_balance_workspace_bytes(ctypes.byref(desc), ctypes.byref(n)),
           "prism_balance_workspace_bytes")
    return torch.empty(n.value, dtype=torch.uint8, device=device)


def _typed(t: Optional[torch.Tensor], dtype: torch.dtype, shape: tuple, dev: int, what: str) -> Optional[int]:
    """The address of a tensor that has to be of this type and shape, on device `dev`, which the call is enqueued on."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape:
        raise PrismError(f"{what} has to be {dtype} {shape}, not {t.dtype} {tuple(t.shape)}")
    if t.get_device() != dev:
        raise PrismError(f"{what} is on {t.device}, not on the current device")
    if not t.is_contiguous():
        raise PrismError(f"{what} has to be contiguous")
    return t.data_ptr()


def _bytes_on(t: torch.Tensor, dev: int, what: str) -> int:
    """The address of a buffer of bytes on device `dev`."""
    if t.get_device() != dev or not t.is_contiguous():
        raise PrismError(f"{what} has to be a contiguous buffer on the current device")
    return t.data_ptr()


@dataclass
class BalanceOut:
    loss: torch.Tensor          # [G]
    counts: torch.Tensor        # [G, E]
    probs: torch.Tensor         # [G, E]
    n_tokens: torch.Tensor      # [G]


def _balance_groups(T: int, group_tokens: int) -> int:
    return -(-T // group_tokens) if group_tokens > 0 else 1


def prism_balance_loss(desc: LayerDesc, logits, topk_idx, workspace, token_mask=None, group_tokens: int = 0,
                       outputs: Optional[BalanceOut] = None, stream=None) -> BalanceOut:
    """Balance loss, activation counts and mean probabilities of every group of tokens (see prism.h).

    logits [T, E] and topk_idx [T, k] as prism_route returns them; token_mask [T] uint8, 0 for padding."""
    T, E, k = logits.shape[0], desc.n_experts, desc.top_k
    G = _balance_groups(T, group_tokens)
    f32, i32 = torch.float32, torch.int32
    dev = torch.cuda.current_device()
    inputs = (_typed(logits, f32, (T, E), dev, "logits"), _typed(topk_idx, i32, (T, k), dev, "topk_idx"),
              _typed(token_mask, torch.uint8, (T,), dev, "token_mask"))
    o = outputs
    if o is None:
        new = _new_on(stream, logits)
        o = BalanceOut(new((G,)), new((G, E), dtype=i32), new((G, E)), new((G,), dtype=i32))
        made = o.loss.data_ptr(), o.counts.data_ptr(), o.probs.data_ptr(), o.n_tokens.data_ptr()
    else:
        made = (_typed(o.loss, f32, (G,), dev, "loss"), _typed(o.counts, i32, (G, E), dev, "counts"),
                _typed(o.probs, f32, (G, E), dev, "probs"), _typed(o.n_tokens, i32, (G,), dev, "n_tokens"))
    if G == 0:                  # no tokens, no groups: nothing to address
        return o
    _check(load_library().prism_balance_loss(
        ctypes.byref(desc), *inputs, group_tokens, T, *made, _bytes_on(workspace, dev, "workspace"), workspace.numel(),
        _stream_on(dev, stream)), "prism_balance_loss")
    return o


def prism_route_backward(desc: LayerDesc, logits, topk_idx, balance: Optional[BalanceOut] = None, d_loss=None,
                         d_gate=None, token_mask=None, group_tokens: int = 0, d_logits=None,
                         stream=None) -> torch.Tensor:
    """Gradient of sum(d_loss * balance.loss) + sum(d_gate * topk_gate) with respect to the logits (see prism.h)."""
    T, E, k = logits.shape[0], desc.n_experts, desc.top_k
    G = _balance_groups(T, group_tokens)
    f32, i32 = torch.float32, torch.int32
    if (balance is None) != (d_loss is None):
        raise PrismError("d_loss comes with the balance it is the gradient of")
    dev = torch.cuda.current_device()
    logits_ptr = _typed(logits, f32, (T, E), dev, "logits")
    if d_logits is None:
        d_logits = _new_on(stream, logits)((T, E))
        d_ptr = d_logits.data_ptr()
    else:
        d_ptr = _typed(d_logits, f32, (T, E), dev, "d_logits")
    if T == 0:
        return d_logits
    _check(load_library().prism_route_backward(
        ctypes.byref(desc), logits_ptr, _typed(topk_idx, i32, (T, k), dev, "topk_idx"),
        _typed(token_mask, torch.uint8, (T,), dev, "token_mask"), group_tokens, T,
        None if balance is None else _typed(balance.counts, i32, (G, E), dev, "counts"),
        None if balance is None else _typed(balance.n_tokens, i32, (G,), dev, "n_tokens"),
        _typed(d_loss, f32, (G,), dev, "d_loss"), _typed(d_gate, f32, (T, k), dev, "d_gate"),
        d_ptr, _stream_on(dev, stream)), "prism_route_backward")
    return d_logits


@dataclass
class DispatchOut:
    local_src: torch.Tensor
    local_offsets: torch.Tensor
    remote_src: torch.Tensor
    remote_offsets: torch.Tensor
    n_local_remote: torch.Tensor
    remote_bytes: torch.Tensor


def prism_dispatch(desc: LayerDesc, topk_idx, local_mask, workspace, stream=None) -> DispatchOut:
    T, E, k = topk_idx.shape[0], desc.n_experts, desc.top_k
    dev = topk_idx.device
    i32 = dict(dtype=torch.int32, device=dev)
    with _memory_of(stream):
        src = torch.full((2, T * k), -1, **i32)     # one fill for both lists
        out = DispatchOut(src[0], torch.empty((E + 1,), **i32), src[1], torch.empty((E + 1,), **i32),
                          torch.empty((2,), **i32), torch.empty((2,), dtype=torch.int64, device=dev))
    _check(load_library().prism_dispatch(ctypes.byref(desc), _ptr(topk_idx), _ptr(local_mask), T,
                                         _ptr(out.local_src), _ptr(out.local_offsets),
                                         _ptr(out.remote_src), _ptr(out.remote_offsets),
                                         _ptr(out.n_local_remote), _ptr(out.remote_bytes),
                                         _ptr(workspace), workspace.numel(), _stream(stream)),
           "prism_dispatch")
    return out


def _clear_rows(desc: LayerDesc, offsets, n_rows, rows, stream) -> None:
    _check(load_library().prism_clear_rows(ctypes.byref(desc), _ptr(offsets), n_rows, _ptr(rows), _stream(stream)),
           "prism_clear_rows")


def prism_expert_ffn(desc: LayerDesc, x, weights: WeightTable, local_src, local_offsets, workspace,
                     y=None, stream=None) -> torch.Tensor:
    T = x.shape[0]
    rows = T * desc.top_k + desc.n_shared * T
    if y is None:
        y = _new_on(stream, x)((rows, desc.hidden), dtype=torch_dtype(desc))
        _clear_rows(desc, local_offsets, T * desc.top_k, y, stream)
    _check(load_library().prism_expert_ffn(ctypes.byref(desc), _ptr(x), weights.struct_for(desc),
                                           _ptr(local_src), _ptr(local_offsets), T, _ptr(y),
                                           _ptr(workspace), workspace.numel(), _stream(stream)),
           "prism_expert_ffn")
    return y


def prism_combine(desc: LayerDesc, y, local_src, local_offsets, topk_gate, workspace, out=None,
                  stream=None) -> torch.Tensor:
    T = topk_gate.shape[0]
    if out is None:
        out = _new_on(stream, y)((T, desc.hidden), dtype=torch_dtype(desc))
    _check(load_library().prism_combine(ctypes.byref(desc), _ptr(y), _ptr(local_src),
                                        _ptr(local_offsets), _ptr(topk_gate), T, _ptr(out),
                                        _ptr(workspace), workspace.numel(), _stream(stream)),
           "prism_combine")
    return out


@dataclass
class LayerOut:
    out: torch.Tensor
    topk_idx: torch.Tensor
    topk_gate: torch.Tensor
    counts: torch.Tensor
    remote_src: torch.Tensor
    remote_offsets: torch.Tensor
    n_local_remote: torch.Tensor
    remote_bytes: torch.Tensor


def alloc_layer_out(desc: LayerDesc, T: int, device="cuda") -> LayerOut:
    E, k = desc.n_experts, desc.top_k
    i32 = dict(dtype=torch.int32, device=device)
    return LayerOut(torch.empty((T, desc.hidden), dtype=torch_dtype(desc), device=device),
                    torch.empty((T, k), **i32), torch.empty((T, k), dtype=torch.float32, device=device),
                    torch.empty((E,), **i32), torch.full((T * k,), -1, **i32),
                    torch.empty((E + 1,), **i32), torch.empty((2,), **i32),
                    torch.empty((2,), dtype=torch.int64, device=device))


def prism_moe_layer(desc: LayerDesc, x, w_router, router_bias, weights: WeightTable, local_mask,
                    workspace, outputs: Optional[LayerOut] = None, counts_accum=None,
                    stream=None, stage_events=None) -> LayerOut:
    """stage_events: optional ctypes array of 2*len(STAGES) hipEvent_t handles (see prism.h)."""
    T = x.shape[0]
    o = outputs
    if o is None:
        with _memory_of(stream):
            o = alloc_layer_out(desc, T, x.device)
    lib = load_library()
    if stage_events is not None:
        _check(lib.prism_moe_layer_traced(ctypes.byref(desc), _ptr(x), _ptr(w_router),
                                          _ptr(router_bias), weights.struct_for(desc),
                                          _ptr(local_mask), T, _ptr(o.out), _ptr(o.topk_idx),
                                          _ptr(o.topk_gate), _ptr(o.counts), _ptr(counts_accum),
                                          _ptr(o.remote_src), _ptr(o.remote_offsets),
                                          _ptr(o.n_local_remote), _ptr(o.remote_bytes),
                                          _ptr(workspace), workspace.numel(), _stream(stream),
                                          ctypes.cast(stage_events, ctypes.c_void_p)),
               "prism_moe_layer_traced")
        return o
    _check(load_library().prism_moe_layer(ctypes.byref(desc), _ptr(x), _ptr(w_router),
                                          _ptr(router_bias), weights.struct_for(desc),
                                          _ptr(local_mask), T, _ptr(o.out), _ptr(o.topk_idx),
                                          _ptr(o.topk_gate), _ptr(o.counts), _ptr(counts_accum),
                                          _ptr(o.remote_src), _ptr(o.remote_offsets),
                                          _ptr(o.n_local_remote), _ptr(o.remote_bytes),
                                          _ptr(workspace), workspace.numel(), _stream(stream)),
           "prism_moe_layer")
    return o


STATIC_SCRATCH_BYTES = 32 << 20


def prism_moe_layer_static(desc: LayerDesc, x, w_router, router_bias, weights: WeightTable, local_mask,
                           outputs: LayerOut, counts_accum=None, stream=None) -> LayerOut:
    """The layer on the library's fixed scratch array: no workspace, nothing allocated (the caller
    supplies every output buffer)."""
    o = outputs
    _check(load_library().prism_moe_layer_static(ctypes.byref(desc), _ptr(x), _ptr(w_router),
                                                 _ptr(router_bias), weights.struct_for(desc),
                                                 _ptr(local_mask), x.shape[0], _ptr(o.out),
                                                 _ptr(o.topk_idx), _ptr(o.topk_gate), _ptr(o.counts),
                                                 _ptr(counts_accum), _ptr(o.remote_src),
                                                 _ptr(o.remote_offsets), _ptr(o.n_local_remote),
                                                 _ptr(o.remote_bytes), _stream(stream)),
           "prism_moe_layer_static")
    return o


@dataclass
class LayerPermutation:
    local_src: torch.Tensor
    local_offsets: torch.Tensor
    inv: torch.Tensor


def prism_layer_permutation(desc: LayerDesc, T: int, workspace, stream=None) -> LayerPermutation:
    """Copies of the permutation the last whole-layer call left in `workspace` (see prism.h)."""
    i32 = dict(dtype=torch.int32, device=workspace.device)
    A = T * desc.top_k
    with _memory_of(stream):
        p = LayerPermutation(torch.full((A,), -1, **i32), torch.empty((desc.n_experts + 1,), **i32),
                             torch.empty((A,), **i32))
    _check(load_library().prism_layer_permutation(ctypes.byref(desc), T, _ptr(workspace),
                                                  workspace.numel(), _ptr(p.local_src),
                                                  _ptr(p.local_offsets), _ptr(p.inv), _stream(stream)),
           "prism_layer_permutation")
    return p


def prism_ceiling_mfma_bf16(operands, out, n_workgroups: int, iters: int, stream=None) -> float:
    """Enqueues the pure-MFMA loop (see prism.h); returns the flop count of the launch."""
    flop = ctypes.c_double(0.0)
    _check(load_library().prism_ceiling_mfma_bf16(_ptr(operands), _ptr(out), n_workgroups, iters,
                                                  ctypes.byref(flop), _stream(stream)),
           "prism_ceiling_mfma_bf16")
    return flop.value


def prism_ceiling_hbm_read(src, out, n_workgroups: int, stream=None) -> int:
    """Enqueues the streaming read of all of src (see prism.h); returns the bytes read."""
    nbytes = src.numel() * src.element_size()
    _check(load_library().prism_ceiling_hbm_read(_ptr(src), ctypes.c_size_t(nbytes), _ptr(out),
                                                 n_workgroups, _stream(stream)),
           "prism_ceiling_hbm_read")
    return nbytes // 16 * 16


def prism_ceiling_hbm_read_pattern(src, out, n_workgroups: int, loads_in_flight: int, span_bytes: int,
                                   mode: int, stream=None) -> int:
    """Enqueues the streaming read with the given access pattern (see prism.h); returns the bytes read."""
    n = ctypes.c_size_t(0)
    _check(load_library().prism_ceiling_hbm_read_pattern(_ptr(src), ctypes.c_size_t(src.numel() * src.element_size()),
                                                         _ptr(out), n_workgroups, loads_in_flight,
                                                         ctypes.c_size_t(span_bytes), mode, ctypes.byref(n),
                                                         _stream(stream)),
           "prism_ceiling_hbm_read_pattern")
    return n.value


def prism_pack_remote(desc: LayerDesc, x, remote_src, remote_offsets, stream=None) -> torch.Tensor:
    """Activation rows to ship, in remote-list order ([T*k, H]; rows past the remote count are zero)."""
    T = x.shape[0]
    packed = _new_on(stream, x)((T * desc.top_k, desc.hidden))
    _clear_rows(desc, remote_offsets, T * desc.top_k, packed, stream)
    _check(load_library().prism_pack_remote(ctypes.byref(desc), _ptr(x), _ptr(remote_src),
                                            _ptr(remote_offsets), T, _ptr(packed), _stream(stream)),
           "prism_pack_remote")
    return packed


def prism_combine_remote(desc: LayerDesc, y_remote, remote_src, remote_offsets, topk_gate, out,
                         workspace, stream=None) -> torch.Tensor:
    """Adds the returned expert outputs (remote-list order) into out, in place."""
    T = topk_gate.shape[0]
    _check(load_library().prism_combine_remote(ctypes.byref(desc), _ptr(y_remote), _ptr(remote_src),
                                               _ptr(remote_offsets), _ptr(topk_gate), T, _ptr(out),
                                               _ptr(workspace), workspace.numel(), _stream(stream)),
           "prism_combine_remote")
    return out


def prism_debug_check_weights(desc: LayerDesc, weights: WeightTable, local_mask) -> None:
    """Blocking check that every hosted and every shared expert has usable weight pointers."""
    bad = ctypes.c_int32(-1)
    code = load_library().prism_debug_check_weights(ctypes.byref(desc), weights.struct_for(desc),
                                                    _ptr(local_mask), ctypes.byref(bad))
    if code != 0:
        what = f"expert {bad.value}" if bad.value >= 0 else "arguments"
        _check(code, f"prism_debug_check_weights ({what})")


def prism_pack_weights(w, stream=None) -> torch.Tensor:
    """Row-major bf16 weight matrix -> the layout of 16 x 32 tiles (a new tensor of the same shape)."""
    rows, cols = w.shape
    packed = _new_on(stream, w)((rows, cols))
    _check(load_library().prism_pack_weights(_ptr(w), rows, cols, _ptr(packed), _stream(stream)),
           "prism_pack_weights")
    return packed


@dataclass
class I8Matrix:
    """A matrix in 8 bits with a scale per row, in the library's layout (prism.h, "8-bit matrices")."""
    data: torch.Tensor          # bytes
    rows: int
    cols: int

    def __post_init__(self):
        if self.data.numel() * self.data.element_size() < _i8_bytes(self.rows, self.cols):
            raise PrismError(f"{self.data.numel()} bytes are too few for an 8-bit matrix of {self.rows} x {self.cols}")

    def values(self):
        """(int8 [rows, cols], scales [rows]): copies in plain order."""
        R, C = -(-self.rows // 16) * 16, -(-self.cols // 128) * 128
        q = self.data[:R * C].view(torch.int8).view(R // 16, C // 64, 16, 64).permute(0, 2, 1, 3).reshape(R, C)
        return (q[:self.rows, :self.cols].contiguous(),
                self.data[R * C:R * C + 4 * self.rows].clone().view(torch.float32))


def _i8_bytes(rows: int, cols: int) -> int:
    """prism_i8_bytes, for sizes that the call the buffer is for will check."""
    R = -(-rows // 16) * 16
    return -(-(R * (-(-cols // 128) * 128) + 4 * R) // 256) * 256


def _rows_ptr(t: torch.Tensor, dev: int, what: str):
    """(address, elements from row to row) of a matrix on device `dev` whose rows are contiguous."""
    if t.dim() != 2:
        raise PrismError(f"{what} has to be a matrix")
    if t.get_device() != dev:
        raise PrismError(f"{what} is on {t.device}, not on the current device")
    rows, cols = t.shape
    ld = cols
    if not t.is_contiguous():
        ld, step = t.stride()
        if rows <= 1:
            ld = cols
        if cols > 1 and step != 1 or ld < cols:
            raise PrismError(f"{what} has to have contiguous rows that do not overlap")
    return t.data_ptr(), ld


_FLOAT_DTYPES = {torch.float32: PRISM_F32, torch.bfloat16: PRISM_BF16}


def _float_dtype(t: torch.Tensor, what: str) -> int:
    if t.dtype not in _FLOAT_DTYPES:
        raise PrismError(f"{what} has to be fp32 or bf16, not {t.dtype}")
    return _FLOAT_DTYPES[t.dtype]


def _out_i8(out: Optional[I8Matrix], rows: int, cols: int, like: torch.Tensor, stream) -> I8Matrix:
    if out is None:
        return I8Matrix(_new_on(stream, like)((_i8_bytes(rows, cols),), dtype=torch.uint8), rows, cols)
    if (out.rows, out.cols) != (rows, cols):
        raise PrismError(f"out is an 8-bit matrix of {out.rows} x {out.cols}, not {rows} x {cols}")
    return out


def prism_quantize_i8(src, out: Optional[I8Matrix] = None, stream=None) -> I8Matrix:
    """fp32 or bf16 rows -> 8 bits with a scale per row (see prism.h)."""
    dev = torch.cuda.current_device()
    dtype = _float_dtype(src, "src")
    ptr, ld = _rows_ptr(src, dev, "src")
    rows, cols = src.shape
    o = _out_i8(out, rows, cols, src, stream)
    _check(load_library().prism_quantize_i8(ptr, dtype, ld, rows, cols, _bytes_on(o.data, dev, "out"), _stream_on(dev, stream)),
           "prism_quantize_i8")
    return o


def prism_pack_i8(q, scale, out: Optional[I8Matrix] = None, stream=None) -> I8Matrix:
    """int8 rows and their fp32 scales, as a checkpoint holds them -> the library's layout."""
    dev = torch.cuda.current_device()
    if q.dtype != torch.int8:
        raise PrismError(f"q has to be int8, not {q.dtype}")
    ptr, ld = _rows_ptr(q, dev, "q")
    rows, cols = q.shape
    o = _out_i8(out, rows, cols, q, stream)
    _check(load_library().prism_pack_i8(ptr, ld, _typed(scale, torch.float32, (rows,), dev, "scale"), rows, cols,
                                        _bytes_on(o.data, dev, "out"), _stream_on(dev, stream)), "prism_pack_i8")
    return o


def alloc_matmul_i8_workspace(max_m: int, n: int, k: int, device="cuda") -> torch.Tensor:
    b = ctypes.c_size_t(0)
    _check(load_library().prism_matmul_i8_workspace_bytes(max_m, n, k, ctypes.byref(b)), "prism_matmul_i8_workspace_bytes")
    return torch.empty(b.value, dtype=torch.uint8, device=device)


def prism_matmul_i8(a: I8Matrix, b: I8Matrix, workspace, out=None, dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """a b^T of two 8-bit matrices [m, k] and [n, k]: [m, n] in bf16 or fp32."""
    if a.cols != b.cols:
        raise PrismError(f"rows of {a.cols} and of {b.cols} elements")
    dev = torch.cuda.current_device()
    if out is None:
        out = _new_on(stream, b.data)((a.rows, b.rows), dtype=dtype)
        ptr, ldo = out.data_ptr(), b.rows
    else:
        if out.shape != (a.rows, b.rows):
            raise PrismError(f"out has to be {a.rows} x {b.rows}, not {tuple(out.shape)}")
        ptr, ldo = _rows_ptr(out, dev, "out")
    out_dtype = _float_dtype(out, "out")
    _check(load_library().prism_matmul_i8(_bytes_on(a.data, dev, "a"), _bytes_on(b.data, dev, "b"), a.rows, b.rows, a.cols, ptr, ldo,
                                          out_dtype, _bytes_on(workspace, dev, "workspace"), workspace.numel(),
                                          _stream_on(dev, stream)), "prism_matmul_i8")
    return out
