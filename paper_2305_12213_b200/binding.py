"""Thin ctypes binding of libdynbatch (argument marshalling only).

Every function has the name and meaning of the C entry point declared in
include/dynbatch.h; tensors are torch tensors used purely as device memory
(`data_ptr()`), and the stream is torch's current stream unless given.  All
arithmetic runs inside the CUDA library: there is no Python or CPU fallback,
and a missing shared library is an error, not a reason to compute elsewhere.
"""
from __future__ import annotations

import ctypes
import operator
import os
import struct
from ctypes import c_char_p, c_double, c_float, c_int32, c_int64, c_size_t, c_void_p
from typing import Optional, Sequence

import torch

DB_OK, DB_ERR_NULL, DB_ERR_ARG, DB_ERR_UNSUPPORTED, DB_ERR_INFEASIBLE, DB_ERR_CUDA = range(6)
DB_F32, DB_BF16, DB_E4M3 = 0, 1, 2
DB_MAX_K = 64
DB_STATIC_SCRATCH_BYTES = 1 << 20     # the built-in scratch of aggregate_update_static
DB_ADAMW_BLOCK = 256                  # elements that share a scale of an 8-bit moment
DB_ADAMW_CLIP = 1
DB_ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
DB_CHECKPOINT_GROUP = 32              # values of a row that share a scale of an 8-bit checkpoint

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "csrc", "libdynbatch.so")

_lib = None


class DynbatchError(RuntimeError):
    """A libdynbatch call returned a status other than DB_OK."""

    def __init__(self, status: int, message: str):
        super().__init__(f"libdynbatch status {status}: {message}")
        self.status = status


_SIGNATURES = {
    "db_aggregate_update": (c_int32, [c_void_p, c_void_p, c_int32, c_int64, c_void_p, c_void_p,
                                      c_float, c_float]),
    "db_aggregate_update_ex": (c_int32, [c_void_p, c_int32, c_void_p, c_int32, c_int64, c_void_p,
                                         c_void_p, c_float, c_float, c_void_p, c_void_p, c_size_t,
                                         c_void_p]),
    "db_aggregate_workspace_bytes": (c_size_t, [c_int32, c_int64]),
    "db_aggregate_adam_ex": (c_int32, [c_void_p, c_int32, c_void_p, c_int32, c_int64, c_void_p, c_void_p, c_void_p,
                                       c_float, c_float, c_float, c_float, c_int64, c_void_p, c_void_p, c_size_t,
                                       c_void_p]),
    "db_multi_plan_device_bytes": (c_size_t, [c_int32, c_int32, c_void_p, c_int32]),
    "db_multi_plan_create": (c_int32, [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_int32, c_void_p, c_void_p,
                                       c_void_p, c_size_t, c_void_p]),
    "db_aggregate_update_multi": (c_int32, [c_void_p, c_void_p, c_float, c_float, c_void_p, c_void_p]),
    "db_multi_plan_destroy": (c_int32, [c_void_p]),
    "db_adamw_plan_device_bytes": (c_size_t, [c_int32, c_int32, c_int32, c_void_p, c_int32, ctypes.c_uint32]),
    "db_adamw_plan_create": (c_int32, [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_int32, c_void_p, c_void_p,
                                       c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_void_p, ctypes.c_uint32,
                                       c_void_p, c_size_t, c_void_p]),
    "db_aggregate_adamw_multi": (c_int32, [c_void_p, c_void_p, c_float, c_float, c_float, c_float, c_int64, c_float,
                                           ctypes.c_uint64, c_void_p, c_void_p]),
    "db_adamw_plan_destroy": (c_int32, [c_void_p]),
    "db_grad_norm_plan_device_bytes": (c_size_t, [c_int32, c_int32, c_void_p, c_int32]),
    "db_grad_norm_plan_create": (c_int32, [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_int32, c_void_p, c_size_t,
                                           c_void_p]),
    "db_grad_norm_multi": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p]),
    "db_grad_norm_plan_destroy": (c_int32, [c_void_p]),
    "db_aggregate_update_static": (c_int32, [c_void_p, c_int32, c_void_p, c_int32, c_int64, c_void_p,
                                             c_void_p, c_float, c_float, c_void_p, c_void_p]),
    "db_shard_range": (c_int32, [c_int64, c_int32, c_int32, c_int32, c_void_p, c_void_p]),
    "db_bench_read_probe_sink_bytes": (c_size_t, [c_size_t]),
    "db_bench_read_probe": (c_int32, [c_void_p, c_size_t, c_void_p, c_void_p]),
    "db_bench_wait_timeout": (c_int32, [c_void_p, c_int32, ctypes.c_uint64, c_void_p]),
    "db_bench_layer_plan": (c_int32, [c_int32, c_int64, c_int32, c_int32, c_void_p, c_void_p, c_void_p]),
    "db_bench_aggregate_variant": (c_int32, [c_int32, c_int32, c_void_p, c_void_p, c_int32, c_int64, c_void_p,
                                             c_void_p, c_float, c_float, c_void_p, c_void_p]),
    "db_host_pipeline_create": (c_int32, [c_void_p]),
    "db_host_pipeline_destroy": (c_int32, [c_void_p]),
    "db_host_staging_bytes": (c_size_t, [c_int32, c_int32, c_int64, c_int64]),
    "db_aggregate_update_host": (c_int32, [c_void_p, c_void_p, c_int32, c_void_p, c_int32, c_int64, c_void_p,
                                           c_void_p, c_float, c_float, c_void_p, c_void_p, c_void_p, c_size_t,
                                           c_int64, c_void_p]),
    "db_worker_grad": (c_int32, [c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p,
                                 c_void_p, c_void_p, c_size_t, c_void_p]),
    "db_worker_grad_ex": (c_int32, [c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p,
                                    c_void_p, c_void_p, c_size_t, ctypes.c_uint32, c_void_p]),
    "db_worker_grad_grouped": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_int32,
                                         c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]),
    "db_worker_grad_grouped_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32, c_int32]),
    "db_contract_f32": (c_int32, [c_void_p, c_int64, c_int64, c_void_p, c_int64, c_int64, c_void_p, c_int64,
                                  c_int64, c_int32, c_int32, c_int32, c_void_p, c_void_p]),
    "db_worker_grad_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32]),
    "db_controller_step": (c_int32, [c_void_p, c_void_p, c_int32, c_double]),
    "db_controller_step_ex": (c_int32, [c_void_p, c_void_p, c_int32, c_double, c_void_p, c_void_p]),
    "db_static_allocate": (c_int32, [c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p]),
    "db_controller_create": (c_int32, [c_void_p, c_void_p, c_int32, c_double, c_double, c_double, c_void_p,
                                       c_void_p, c_int32]),
    "db_controller_observe": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p]),
    "db_controller_destroy": (c_int32, [c_void_p]),
    "db_linear_workspace_bytes": (c_size_t, [c_int64, c_int32, c_int32, c_int32]),
    "db_linear": (c_int32, [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_int64, c_int32, c_int32,
                            c_void_p, c_int64, c_void_p, c_void_p, c_int32, c_void_p, c_size_t, c_void_p]),
    "db_linear_grad_workspace_bytes": (c_size_t, [c_int64, c_int32, c_int32, c_int32]),
    "db_linear_grad": (c_int32, [c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int32, c_int32,
                                 c_int64, c_int32, c_int32, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p,
                                 c_int32, c_void_p, c_size_t, c_void_p]),
    "db_gated_ffn_workspace_bytes": (c_size_t, [c_int64, c_int32, c_int32, c_int32]),
    "db_gated_ffn": (c_int32, [c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_int32, c_int64,
                               c_int32, c_int32, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_int32,
                               c_void_p, c_size_t, c_void_p]),
    "db_gated_ffn_grad_workspace_bytes": (c_size_t, [c_int64, c_int32, c_int32, c_int32]),
    "db_gated_ffn_grad": (c_int32, [c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                    c_void_p, c_void_p, c_int32, c_int32, c_int64, c_int32, c_int32, c_void_p, c_int64,
                                    c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int32, c_void_p, c_size_t,
                                    c_void_p]),
    "db_checkpoint_pack": (c_int32, [c_void_p, c_int64, c_int64, c_int32, c_void_p, c_void_p, c_void_p]),
    "db_checkpoint_unpack": (c_int32, [c_void_p, c_void_p, c_int64, c_int32, c_void_p, c_int64, c_void_p]),
    "db_embedding": (c_int32, [c_void_p, c_void_p, c_int32, c_float, c_int64, c_int32, c_int32, c_void_p, c_int64, c_int32,
                               c_void_p]),
    "db_embedding_grad_workspace_bytes": (c_size_t, [c_int64, c_int32, c_int32]),
    "db_embedding_grad": (c_int32, [c_void_p, c_void_p, c_int64, c_int32, c_float, c_int64, c_int32, c_int32, c_void_p,
                                    c_int32, c_void_p, c_size_t, c_void_p]),
    "db_status_string": (c_char_p, [c_int32]),
    "db_last_cuda_error": (c_char_p, []),
}


def lib() -> ctypes.CDLL:
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2305_12213_b200.build`. "
                "libdynbatch has no CPU fallback.")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != DB_OK:
        L = lib()
        msg = L.db_status_string(status).decode()
        if status in (DB_ERR_CUDA, DB_ERR_UNSUPPORTED):
            detail = L.db_last_cuda_error().decode()
            if detail:
                msg += ": " + detail
        raise DynbatchError(status, msg)


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _i32_array(values: Sequence[int]):
    return (c_int32 * len(values))(*[int(x) for x in values])


def _dev_ptr(t: Optional[torch.Tensor], dtype: torch.dtype, name: str) -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous CUDA tensor of {dtype}")
    return t.data_ptr()


def aggregate_workspace_bytes(K: int, N: int) -> int:
    return int(lib().db_aggregate_workspace_bytes(int(K), int(N)))


def aggregate_update(grads: Sequence[torch.Tensor], b: Sequence[int], params: torch.Tensor,
                     momentum: torch.Tensor, lr: float, mu: float,
                     grad_sqnorm: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None, N: Optional[int] = None) -> None:
    """db_aggregate_update_ex: fused weighted aggregation + momentum-SGD update, in place.

    grads: K CUDA tensors (all float32 or all bfloat16) of N elements; b: K batch sizes;
    params, momentum: float32 CUDA tensors; grad_sqnorm: optional float64 CUDA tensor of one
    element; workspace: uint8 CUDA tensor of aggregate_workspace_bytes(K, N) when the norm is wanted.
    """
    K = len(grads)
    if len(b) != K:
        raise ValueError("len(b) != len(grads)")
    gdt = grads[0].dtype
    if gdt == torch.float32:
        code = DB_F32
    elif gdt == torch.bfloat16:
        code = DB_BF16
    else:
        raise TypeError("gradients must be float32 or bfloat16")
    n = int(params.numel() if N is None else N)
    table = (c_void_p * K)(*[_dev_ptr(g, gdt, "grads[k]") for g in grads])
    _check(lib().db_aggregate_update_ex(
        ctypes.cast(table, c_void_p), code, ctypes.cast(_i32_array(b), c_void_p), K, n,
        _dev_ptr(params, torch.float32, "params"), _dev_ptr(momentum, torch.float32, "momentum"),
        float(lr), float(mu), _dev_ptr(grad_sqnorm, torch.float64, "grad_sqnorm"),
        None if workspace is None else workspace.data_ptr(),
        0 if workspace is None else workspace.numel() * workspace.element_size(),
        _stream_ptr(stream)))


class AggregateStep:
    """db_aggregate_update_ex with its tensor arguments marshalled once: for loops that call the step
    on the same buffers every iteration (the pointers, not the tensors' contents, are fixed here).
    `run(b, lr, mu)` then only converts the batch sizes and the two scalars."""

    def __init__(self, grads: Sequence[torch.Tensor], params: torch.Tensor, momentum: torch.Tensor,
                 grad_sqnorm: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None):
        self.K = len(grads)
        gdt = grads[0].dtype
        if gdt not in (torch.float32, torch.bfloat16):
            raise TypeError("gradients must be float32 or bfloat16")
        self._keep = (list(grads), params, momentum, grad_sqnorm, workspace)       # the buffers stay alive
        self._table = (c_void_p * self.K)(*[_dev_ptr(g, gdt, "grads[k]") for g in grads])
        self._b = (c_int32 * self.K)()
        self._fn = lib().db_aggregate_update_ex
        self._args = (ctypes.cast(self._table, c_void_p), DB_F32 if gdt == torch.float32 else DB_BF16,
                      ctypes.cast(self._b, c_void_p), self.K, int(params.numel()),
                      _dev_ptr(params, torch.float32, "params"), _dev_ptr(momentum, torch.float32, "momentum"))
        self._tail = (_dev_ptr(grad_sqnorm, torch.float64, "grad_sqnorm"),
                      None if workspace is None else workspace.data_ptr(),
                      0 if workspace is None else workspace.numel() * workspace.element_size(),
                      _stream_ptr(stream))

    def run(self, b: Sequence[int], lr: float, mu: float) -> None:
        if len(b) != self.K:
            raise ValueError("len(b) != number of gradient buffers")
        self._b[:] = b
        _check(self._fn(*self._args, lr, mu, *self._tail))


def aggregate_adam(grads: Sequence[torch.Tensor], b: Sequence[int], params: torch.Tensor,
                   first_moment: torch.Tensor, second_moment: torch.Tensor, lr: float, beta1: float,
                   beta2: float, eps: float, step: int, grad_sqnorm: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_aggregate_adam_ex: fused weighted aggregation + Adam update (bias-corrected), in place."""
    K = len(grads)
    if len(b) != K:
        raise ValueError("len(b) != len(grads)")
    gdt = grads[0].dtype
    table = (c_void_p * K)(*[_dev_ptr(g, gdt, "grads[k]") for g in grads])
    code = DB_F32 if gdt == torch.float32 else DB_BF16 if gdt == torch.bfloat16 else -1
    _check(lib().db_aggregate_adam_ex(
        ctypes.cast(table, c_void_p), code, ctypes.cast(_i32_array(b), c_void_p), K, int(params.numel()),
        _dev_ptr(params, torch.float32, "params"), _dev_ptr(first_moment, torch.float32, "first_moment"),
        _dev_ptr(second_moment, torch.float32, "second_moment"), float(lr), float(beta1), float(beta2),
        float(eps), int(step), _dev_ptr(grad_sqnorm, torch.float64, "grad_sqnorm"),
        None if workspace is None else workspace.data_ptr(),
        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream_ptr(stream)))


def aggregate_update_static(grads: Sequence[torch.Tensor], b: Sequence[int], params: torch.Tensor,
                            momentum: torch.Tensor, lr: float, mu: float,
                            grad_sqnorm: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_aggregate_update_static: aggregate_update for callers that cannot supply a workspace.

    The norm's scratch is a fixed array inside the library, shared by every call on the device, so
    calls that could overlap on the GPU must be serialised by the caller.  Nothing is allocated.
    """
    K = len(grads)
    if len(b) != K:
        raise ValueError("len(b) != len(grads)")
    gdt = grads[0].dtype
    if gdt not in (torch.float32, torch.bfloat16):
        raise TypeError("gradients must be float32 or bfloat16")
    table = (c_void_p * K)(*[_dev_ptr(g, gdt, "grads[k]") for g in grads])
    _check(lib().db_aggregate_update_static(
        ctypes.cast(table, c_void_p), DB_F32 if gdt == torch.float32 else DB_BF16,
        ctypes.cast(_i32_array(b), c_void_p), K, int(params.numel()),
        _dev_ptr(params, torch.float32, "params"), _dev_ptr(momentum, torch.float32, "momentum"),
        float(lr), float(mu), _dev_ptr(grad_sqnorm, torch.float64, "grad_sqnorm"), _stream_ptr(stream)))


def shard_range(N: int, G: int, r: int, align: int = 8):
    """db_shard_range: the slice [begin, end) of N parameters that parameter server r of G owns."""
    lo, hi = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(lib().db_shard_range(int(N), int(G), int(r), int(align), ctypes.byref(lo), ctypes.byref(hi)))
    return int(lo.value), int(hi.value)


DB_BENCH_PERSISTENT, DB_BENCH_BULK_STAGED = 1, 2


def bench_read_probe_sink_bytes(nbytes: int) -> int:
    return int(lib().db_bench_read_probe_sink_bytes(int(nbytes)))


def bench_read_probe(src: torch.Tensor, sink: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_bench_read_probe: stream all of `src` through registers once (a measurement helper)."""
    if not (src.is_cuda and sink.is_cuda and src.is_contiguous() and sink.is_contiguous()):
        raise TypeError("src and sink must be contiguous CUDA tensors")
    nbytes = src.numel() * src.element_size()
    if sink.numel() * sink.element_size() < bench_read_probe_sink_bytes(nbytes):
        raise ValueError("sink too small")
    _check(lib().db_bench_read_probe(src.data_ptr(), nbytes, sink.data_ptr(), _stream_ptr(stream)))


def bench_wait_timeout(status: torch.Tensor, code: int, limit_ns: int,
                       stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_bench_wait_timeout: run the kernels' bounded wait until it gives up and reports `code`."""
    _check(lib().db_bench_wait_timeout(_dev_ptr(status, torch.int32, "status"), int(code), int(limit_ns),
                                       _stream_ptr(stream)))


DB_BENCH_LAYER_PRODUCTS = {"linear_y": 0, "linear_dx": 1, "linear_dw": 2, "gated_h": 3, "gated_y": 4, "gated_dh": 5,
                           "gated_dx": 6, "gated_dw": 7}


def bench_layer_plan(product: str, rows: int, n_in: int, n_out: int):
    """db_bench_layer_plan: (CTAs that share a tile, columns of a tile, pieces of the reduction) of a layer's product."""
    out = (c_int32 * 3)()
    at = ctypes.addressof(out)
    _check(lib().db_bench_layer_plan(DB_BENCH_LAYER_PRODUCTS[product], int(rows), int(n_in), int(n_out), at, at + 4, at + 8))
    return tuple(out)


def bench_aggregate_variant(variant: int, stage_floats: int, grads: Sequence[torch.Tensor], b: Sequence[int],
                            params: torch.Tensor, momentum: torch.Tensor, lr: float, mu: float,
                            status: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_bench_aggregate_variant: the momentum step in a launch shape that was measured and not adopted."""
    K = len(grads)
    if len(b) != K:
        raise ValueError("len(b) != len(grads)")
    table = (c_void_p * K)(*[_dev_ptr(g, torch.float32, "grads[k]") for g in grads])
    _check(lib().db_bench_aggregate_variant(
        int(variant), int(stage_floats), ctypes.cast(table, c_void_p), ctypes.cast(_i32_array(b), c_void_p), K,
        int(params.numel()), _dev_ptr(params, torch.float32, "params"), _dev_ptr(momentum, torch.float32, "momentum"),
        float(lr), float(mu), _dev_ptr(status, torch.int32, "status"), _stream_ptr(stream)))


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.float32:
        return DB_F32
    if dt == torch.bfloat16:
        return DB_BF16
    raise TypeError("gradients must be float32 or bfloat16")


def host_staging_bytes(K: int, grad_dtype: torch.dtype, N: int, chunk_elems: int = 0) -> int:
    return int(lib().db_host_staging_bytes(int(K), _dtype_code(grad_dtype), int(N), int(chunk_elems)))


class HostPipeline:
    """db_host_pipeline: side streams and events for db_aggregate_update_host on the current device."""

    def __init__(self):
        self._h = c_void_p()
        _check(lib().db_host_pipeline_create(ctypes.byref(self._h)))

    def close(self) -> None:
        if self._h:
            lib().db_host_pipeline_destroy(self._h)
            self._h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def aggregate_update(self, host_grads: Sequence[torch.Tensor], b: Sequence[int], params: torch.Tensor,
                         momentum: torch.Tensor, lr: float, mu: float,
                         host_params_out: Optional[torch.Tensor], host_sqnorm_out: Optional[torch.Tensor],
                         staging: torch.Tensor, chunk_elems: int = 0,
                         stream: Optional[torch.cuda.Stream] = None) -> None:
        """db_aggregate_update_host: gradients in (pinned) host tensors, parameters copied back to the host."""
        K = len(host_grads)
        if len(b) != K:
            raise ValueError("len(b) != len(host_grads)")
        gdt = host_grads[0].dtype
        for g in host_grads:
            if g.is_cuda or g.dtype != gdt or not g.is_contiguous():
                raise TypeError("host_grads must be contiguous CPU tensors of one dtype")
        for t, dt, name in ((host_params_out, torch.float32, "host_params_out"),
                            (host_sqnorm_out, torch.float64, "host_sqnorm_out")):
            if t is not None and (t.is_cuda or t.dtype != dt or not t.is_contiguous()):
                raise TypeError(f"{name} must be a contiguous CPU tensor of {dt}")
        table = (c_void_p * K)(*[g.data_ptr() for g in host_grads])
        _check(lib().db_aggregate_update_host(
            self._h, ctypes.cast(table, c_void_p), _dtype_code(gdt), ctypes.cast(_i32_array(b), c_void_p), K,
            int(params.numel()), _dev_ptr(params, torch.float32, "params"),
            _dev_ptr(momentum, torch.float32, "momentum"), float(lr), float(mu),
            None if host_params_out is None else host_params_out.data_ptr(),
            None if host_sqnorm_out is None else host_sqnorm_out.data_ptr(),
            staging.data_ptr(), staging.numel() * staging.element_size(), int(chunk_elems),
            _stream_ptr(stream)))


def worker_grad_workspace_bytes(b_i: int, D: int, C: int) -> int:
    return int(lib().db_worker_grad_workspace_bytes(int(b_i), int(D), int(C)))


DB_WORKER_GRAD_FFMA = 1


def worker_grad(X: torch.Tensor, y: torch.Tensor, W: torch.Tensor, G: torch.Tensor,
                loss: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None, flags: int = 0) -> None:
    """db_worker_grad_ex: G = X^T (softmax(X W) - onehot(y)) / b_i, optional mean cross-entropy."""
    b_i, D = X.shape
    D2, C = W.shape
    if D2 != D or tuple(G.shape) != (D, C) or y.numel() != b_i:
        raise ValueError("shape mismatch")
    _check(lib().db_worker_grad_ex(
        _dev_ptr(X, torch.float32, "X"), _dev_ptr(y, torch.int32, "y"), _dev_ptr(W, torch.float32, "W"),
        b_i, D, C, _dev_ptr(G, torch.float32, "G"), _dev_ptr(loss, torch.float32, "loss"),
        None if workspace is None else workspace.data_ptr(),
        0 if workspace is None else workspace.numel() * workspace.element_size(),
        int(flags), _stream_ptr(stream)))


def worker_grad_grouped_workspace_bytes(total_rows: int, K: int, D: int, C: int) -> int:
    return int(lib().db_worker_grad_grouped_workspace_bytes(int(total_rows), int(K), int(D), int(C)))


def worker_grad_grouped(X: torch.Tensor, y: torch.Tensor, W: torch.Tensor, offsets: Sequence[int],
                        G: Sequence[torch.Tensor], losses: Optional[torch.Tensor], workspace: torch.Tensor,
                        stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_worker_grad_grouped: every worker's gradient (rows offsets[w]:offsets[w+1] of X, y) in three launches."""
    K = len(G)
    rows, D = X.shape
    D2, C = W.shape
    if len(offsets) != K + 1 or D2 != D or y.numel() != rows or int(offsets[-1]) != rows:
        raise ValueError("shape mismatch")
    for g in G:
        if tuple(g.shape) != (D, C):
            raise ValueError("G[w] must be [D, C]")
    table = (c_void_p * K)(*[_dev_ptr(g, torch.float32, "G[w]") for g in G])
    _check(lib().db_worker_grad_grouped(
        _dev_ptr(X, torch.float32, "X"), _dev_ptr(y, torch.int32, "y"), _dev_ptr(W, torch.float32, "W"),
        ctypes.cast(_i32_array(offsets), c_void_p), K, D, C, ctypes.cast(table, c_void_p),
        _dev_ptr(losses, torch.float32, "losses"), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream_ptr(stream)))


def contract_f32(A: torch.Tensor, B: torch.Tensor, out: torch.Tensor, status: torch.Tensor,
                 stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_contract_f32: out[m, n] = sum_k A[m, k] * B[n, k] for 2-D fp32 CUDA tensors of any strides."""
    M, K = A.shape
    N, K2 = B.shape
    if K2 != K or tuple(out.shape) != (M, N):
        raise ValueError("shape mismatch")
    for t in (A, B, out):
        if not t.is_cuda or t.dtype != torch.float32:
            raise TypeError("A, B, out must be float32 CUDA tensors")
    _check(lib().db_contract_f32(
        A.data_ptr(), A.stride(0), A.stride(1), B.data_ptr(), B.stride(0), B.stride(1), out.data_ptr(),
        out.stride(0), out.stride(1), M, N, K, _dev_ptr(status, torch.int32, "status"), _stream_ptr(stream)))


def worker_grad_status(workspace: torch.Tensor) -> int:
    """The status word at the start of a db_worker_grad workspace (0 = every internal wait completed)."""
    return int(workspace[:4].view(torch.int32).item())


def controller_step(b: Sequence[int], throughputs: Sequence[float], kp: float,
                    b_min: Optional[Sequence[int]] = None,
                    b_max: Optional[Sequence[int]] = None) -> list:
    """db_controller_step_ex: one proportional-control adjustment; returns the new batch sizes."""
    K = len(b)
    if len(throughputs) != K:
        raise ValueError("len(throughputs) != len(b)")
    arr = _i32_array(b)
    xs = (c_double * K)(*[float(x) for x in throughputs])
    lo = None if b_min is None else ctypes.cast(_i32_array(b_min), c_void_p)
    hi = None if b_max is None else ctypes.cast(_i32_array(b_max), c_void_p)
    _check(lib().db_controller_step_ex(ctypes.cast(arr, c_void_p), ctypes.cast(xs, c_void_p), K,
                                       float(kp), lo, hi))
    return list(arr)


def static_allocate(throughputs: Sequence[float], b0: int, b_min: Optional[Sequence[int]] = None,
                    b_max: Optional[Sequence[int]] = None) -> list:
    """db_static_allocate: throughput-proportional batch sizes that keep the global batch K * b0."""
    K = len(throughputs)
    xs = (c_double * K)(*[float(x) for x in throughputs])
    out = (c_int32 * K)()
    lo = None if b_min is None else ctypes.cast(_i32_array(b_min), c_void_p)
    hi = None if b_max is None else ctypes.cast(_i32_array(b_max), c_void_p)
    _check(lib().db_static_allocate(ctypes.cast(xs, c_void_p), K, int(b0), lo, hi, ctypes.cast(out, c_void_p)))
    return list(out)


class Controller:
    """db_controller: the stabilised batch-size controller (EWMA, bounds, dead-band)."""

    def __init__(self, b0: Sequence[int], kp: float = 1.0, alpha: float = 0.5, dead_band: float = 0.05,
                 b_min: Optional[Sequence[int]] = None, b_max: Optional[Sequence[int]] = None,
                 adaptive_b_max: bool = False):
        self.K = len(b0)
        self._h = c_void_p()
        lo = None if b_min is None else ctypes.cast(_i32_array(b_min), c_void_p)
        hi = None if b_max is None else ctypes.cast(_i32_array(b_max), c_void_p)
        _check(lib().db_controller_create(ctypes.byref(self._h), ctypes.cast(_i32_array(b0), c_void_p), self.K,
                                          float(kp), float(alpha), float(dead_band), lo, hi, int(adaptive_b_max)))

    def observe(self, iteration_times: Sequence[float]):
        """Returns (batch sizes in force, whether they were readjusted)."""
        ts = (c_double * self.K)(*[float(t) for t in iteration_times])
        out = (c_int32 * self.K)()
        changed = c_int32(0)
        _check(lib().db_controller_observe(self._h, ctypes.cast(ts, c_void_p), ctypes.cast(out, c_void_p),
                                           ctypes.byref(changed)))
        return list(out), bool(changed.value)

    def close(self) -> None:
        if self._h:
            lib().db_controller_destroy(self._h)
            self._h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class MultiTensorPlan:
    """db_multi_plan: the momentum step over a fixed list of separately allocated tensors.

    grads[k][t] is worker k's gradient of tensor t; params[t], momentum[t] its fp32 state.
    """

    def __init__(self, grads: Sequence[Sequence[torch.Tensor]], params: Sequence[torch.Tensor],
                 momentum: Sequence[torch.Tensor], stream: Optional[torch.cuda.Stream] = None):
        K, T = len(grads), len(params)
        gdt = grads[0][0].dtype
        self.K = K
        sizes = (c_int64 * T)(*[int(p.numel()) for p in params])
        gtab = (c_void_p * (K * T))(*[_dev_ptr(grads[k][t], gdt, "grads[k][t]") for k in range(K) for t in range(T)])
        ptab = (c_void_p * T)(*[_dev_ptr(p, torch.float32, "params[t]") for p in params])
        vtab = (c_void_p * T)(*[_dev_ptr(v, torch.float32, "momentum[t]") for v in momentum])
        for k in range(K):
            for t in range(T):
                if grads[k][t].numel() != params[t].numel():
                    raise ValueError("gradient and parameter sizes differ")
        code = _dtype_code(gdt)
        nbytes = int(lib().db_multi_plan_device_bytes(K, code, ctypes.cast(sizes, c_void_p), T))
        self.table = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=params[0].device)
        self._keep = (list(params), list(momentum), [list(g) for g in grads])   # the plan stores raw pointers
        self._h = c_void_p()
        _check(lib().db_multi_plan_create(ctypes.byref(self._h), ctypes.cast(gtab, c_void_p), code, K,
                                          ctypes.cast(sizes, c_void_p), T, ctypes.cast(ptab, c_void_p),
                                          ctypes.cast(vtab, c_void_p), self.table.data_ptr(), self.table.numel(),
                                          _stream_ptr(stream)))

    def step(self, b: Sequence[int], lr: float, mu: float, grad_sqnorm: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> None:
        """db_aggregate_update_multi: one launch over every tensor of the plan."""
        if len(b) != self.K:
            raise ValueError("len(b) != K")
        _check(lib().db_aggregate_update_multi(self._h, ctypes.cast(_i32_array(b), c_void_p), float(lr), float(mu),
                                               _dev_ptr(grad_sqnorm, torch.float64, "grad_sqnorm"),
                                               _stream_ptr(stream)))

    def close(self) -> None:
        if self._h:
            lib().db_multi_plan_destroy(self._h)
            self._h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _ListPlan:
    """What the plans over a tensor list share: the buffers' device, the worker table and the handle's life."""

    _destroy = ""

    def __init__(self, grads: Sequence[Sequence[torch.Tensor]], shapes: Optional[Sequence[torch.Tensor]]):
        if len(grads) < 1 or len(grads[0]) < 1:
            raise ValueError("at least one worker and one tensor")
        self.K, self.T = len(grads), len(grads[0])
        like = grads[0] if shapes is None else shapes
        if len(like) != self.T or any(len(g) != self.T for g in grads):
            raise ValueError("every worker has one gradient for each tensor")
        self.grad_dtype = grads[0][0].dtype
        self._code = _dtype_code(self.grad_dtype)
        self.device = like[0].device
        self.sizes = [int(t.numel()) for t in like]
        self._sizes = (c_int64 * self.T)(*self.sizes)
        self._keep = []                                  # the plan stores raw pointers: the buffers stay alive
        for g in grads:
            if any(x.numel() != n for x, n in zip(g, self.sizes)):
                raise ValueError("gradient and parameter sizes differ")
        self._grads = (c_void_p * (self.K * self.T))(
            *[p for g in grads for p in self._pointers(g, self.grad_dtype, "grads[k]")])
        self._batches = struct.Struct(f"{self.K}i").pack
        self._h = c_void_p()
        self._streams = set()                            # raw handles of the streams that the table is known to be used on

    def _make_table(self, nbytes: int, stream: Optional[torch.cuda.Stream]) -> None:
        # the allocator may hand out memory that work queued on the current stream still uses
        self.table = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        self._streams.add(torch._C._cuda_getCurrentRawStream(self.device.index))
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream(self.device))

    def _used_on(self, handle: int, stream: Optional[torch.cuda.Stream]) -> None:
        """First use of the table on a stream other than its own: the allocator must not give the memory away before that
        stream is done with it.  (Not while the stream is captured: a graph needs the plan to stay alive anyway.)"""
        s = torch.cuda.current_stream(self.device) if stream is None else stream
        with torch.cuda.stream(s):
            if torch.cuda.is_current_stream_capturing():
                return
        self.table.record_stream(s)
        self._streams.add(handle)

    def _pointers(self, tensors, dtype, name, sizes=None):
        tensors = list(tensors)
        if len(tensors) != self.T:
            raise ValueError(f"{name} must have one tensor for each parameter tensor")
        for t, n in zip(tensors, self.sizes if sizes is None else sizes):
            if t.device != self.device:
                raise ValueError(f"{name}[t] is on {t.device}, the plan's first tensor on {self.device}")
            if t.numel() != n:
                raise ValueError(f"{name}[t] must have {n} elements")
        self._keep.append(tensors)
        return [_dev_ptr(t, dtype, f"{name}[t]") for t in tensors]

    def _array(self, tensors, dtype, name, sizes=None):
        return None if tensors is None else (c_void_p * self.T)(*self._pointers(tensors, dtype, name, sizes))

    def _call(self, fn, *args, stream: Optional[torch.cuda.Stream] = None) -> None:
        """fn(*args, stream) with the plan's device current.  The raw stream handle of that device costs 0.1 us where a
        Stream object costs 2.4, and the switch is left out where the device is current already (another 1.5): small
        models' steps are bound by this side of the call."""
        if stream is not None:
            handle = stream.cuda_stream
        else:
            handle = torch._C._cuda_getCurrentRawStream(self.device.index)
        if handle not in self._streams:
            self._used_on(handle, stream)
        if torch.cuda.current_device() == self.device.index:
            _check(fn(*args, handle))
        else:
            with torch.cuda.device(self.device):
                _check(fn(*args, handle))

    def _workers(self, b: Sequence[int]):
        if len(b) != self.K:
            raise ValueError("len(b) != K")
        # a call's own bytes (another thread's may be under way); a ctypes array would cut its numbers to 32 bits without a
        # word, and making one takes 0.5 us more at two workers, 3 at sixteen
        try:
            return self._batches(*b)
        except struct.error:
            raise ValueError(f"batch sizes beyond 32 bits: {[operator.index(x) for x in b]}") from None

    def _scalar(self, t: Optional[torch.Tensor]) -> Optional[int]:
        if t is not None and (t.device != self.device or t.numel() < 1):
            raise ValueError("grad_norm must hold one element on the plan's device")
        return _dev_ptr(t, torch.float32, "grad_norm")

    def close(self) -> None:
        if self._h:
            getattr(lib(), self._destroy)(self._h)
            self._h = c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class AdamWPlan(_ListPlan):
    """db_adamw_plan: AdamW over a fixed list of tensors, with optional clipping by the global norm.

    grads[k][t] is worker k's gradient of tensor t (all float32 or all bfloat16); params[t] float32;
    first_moment[t], second_moment[t] all float32, or all float8_e4m3fn with first_scale[t], second_scale[t] of
    adamw_scale_elems(numel) float32 elements; params_bf16[t] optional bfloat16 working copies, weight_decay
    one coefficient for each tensor.  clip: whether steps may pass max_norm > 0.
    A CUDA graph that holds a step reads the plan's table at each replay: keep the plan as long as the graph.
    """

    _destroy = "db_adamw_plan_destroy"

    def __init__(self, grads: Sequence[Sequence[torch.Tensor]], params: Sequence[torch.Tensor],
                 first_moment: Sequence[torch.Tensor], second_moment: Sequence[torch.Tensor],
                 first_scale: Optional[Sequence[torch.Tensor]] = None,
                 second_scale: Optional[Sequence[torch.Tensor]] = None,
                 params_bf16: Optional[Sequence[torch.Tensor]] = None,
                 weight_decay: Optional[Sequence[float]] = None, clip: bool = False,
                 stream: Optional[torch.cuda.Stream] = None):
        super().__init__(grads, params)
        if len(first_moment) < 1:
            raise ValueError("first_moment must have one tensor for each parameter tensor")
        state = first_moment[0].dtype
        if state not in (torch.float32, torch.float8_e4m3fn):
            raise TypeError("moments must be float32 or float8_e4m3fn")
        blocks = [adamw_scale_elems(n) for n in self.sizes]
        if weight_decay is not None and len(weight_decay) != self.T:
            raise ValueError("weight_decay must have one coefficient for each parameter tensor")
        p = self._array(params, torch.float32, "params")
        w = self._array(params_bf16, torch.bfloat16, "params_bf16")
        m = self._array(first_moment, state, "first_moment")
        u = self._array(second_moment, state, "second_moment")
        ms = self._array(first_scale, torch.float32, "first_scale", blocks)
        us = self._array(second_scale, torch.float32, "second_scale", blocks)
        wd = None if weight_decay is None else (c_float * self.T)(*[float(x) for x in weight_decay])
        flags = DB_ADAMW_CLIP if clip else 0
        state_code = DB_F32 if state == torch.float32 else DB_E4M3
        nbytes = int(lib().db_adamw_plan_device_bytes(self.K, self._code, state_code, self._sizes, self.T, flags))
        self._make_table(nbytes, stream)
        self._call(lib().db_adamw_plan_create, ctypes.byref(self._h), self._grads, self._code, self.K, self._sizes, self.T,
                   p, w, m, u, state_code, ms, us, wd, flags, self.table.data_ptr(), self.table.numel(), stream=stream)
        self._fn = lib().db_aggregate_adamw_multi

    def step(self, b: Sequence[int], lr: float, beta1: float, beta2: float, eps: float, step: int,
             max_norm: float = 0.0, seed: int = 0, grad_norm: Optional[torch.Tensor] = None,
             stream: Optional[torch.cuda.Stream] = None) -> None:
        """db_aggregate_adamw_multi: one step of every tensor, in place; grad_norm receives the norm before clipping."""
        self._call(self._fn, self._h, self._workers(b), float(lr), float(beta1), float(beta2), float(eps), int(step),
                   float(max_norm), int(seed), self._scalar(grad_norm), stream=stream)


class GradNormPlan(_ListPlan):
    """db_grad_norm_plan: the global norm of the workers' weighted gradient over a fixed list of tensors.  A CUDA graph that
    holds a call reads the plan's table at each replay: keep the plan as long as the graph."""

    _destroy = "db_grad_norm_plan_destroy"

    def __init__(self, grads: Sequence[Sequence[torch.Tensor]], stream: Optional[torch.cuda.Stream] = None):
        super().__init__(grads, None)
        nbytes = int(lib().db_grad_norm_plan_device_bytes(self.K, self._code, self._sizes, self.T))
        self._make_table(nbytes, stream)
        self._call(lib().db_grad_norm_plan_create, ctypes.byref(self._h), self._grads, self._code, self.K, self._sizes,
                   self.T, self.table.data_ptr(), self.table.numel(), stream=stream)
        self._fn = lib().db_grad_norm_multi

    def run(self, b: Sequence[int], grad_norm: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
        """db_grad_norm_multi: grad_norm (one float32) receives the norm."""
        self._call(self._fn, self._h, self._workers(b), self._scalar(grad_norm), stream=stream)


def adamw_scale_elems(n: int) -> int:
    """Scales of an 8-bit moment of n elements: one for each DB_ADAMW_BLOCK."""
    return -(-int(n) // DB_ADAMW_BLOCK)


# ---------------------------------------------------------------------------------------------------------------
# layers.  A call's tensors share one device, which is made current for it.  Small layers' calls are bound by this side
# (a linear layer of 256 rows: 8 us of Python and launch against 10 on the GPU), so the checks ask a tensor each thing once.
# ---------------------------------------------------------------------------------------------------------------
_BF16, _E4M3, _E8M0 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu


def _size(n: int, bits: int = 31) -> int:
    """A size for an int32 (int64: bits = 63) argument, which ctypes would cut to its lowest bits: one past the type's range
    is passed as -1, which every call refuses."""
    return n if 0 <= n >> bits < 1 else -1


def _device_index(first: torch.Tensor) -> int:
    index = first.get_device()
    if index < 0:
        raise TypeError("the tensors of a layer must be CUDA tensors")
    return index


def _elsewhere(t: torch.Tensor, index: int, name: str):
    raise ValueError(f"{name} is on {t.device}, the call's first tensor on cuda:{index}")


def _rows(t: Optional[torch.Tensor], rows: int, cols: int, index: int, name: str, dtype: torch.dtype = _BF16):
    """Pointer and pitch of a [rows, cols] tensor whose rows are contiguous."""
    if t is None:
        return None, 0
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    if t.shape != (rows, cols):
        raise ValueError(f"{name} must be [{rows}, {cols}]")
    if t.get_device() != index:
        _elsewhere(t, index, name)
    pitch, step = t.stride()
    if rows <= 1:
        pitch = cols
    if pitch < cols or (step != 1 and cols > 1):
        raise ValueError(f"the rows of {name} must be contiguous and may not overlap")
    return t.data_ptr(), pitch


def _whole(t: Optional[torch.Tensor], shape, dtype: torch.dtype, index: int, name: str) -> Optional[int]:
    """Pointer of a contiguous tensor."""
    if t is None:
        return None
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}")
    if t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous CUDA tensor of {dtype}")
    if t.get_device() != index:
        _elsewhere(t, index, name)
    return t.data_ptr()


def _kept(t: Optional[torch.Tensor], scale: Optional[torch.Tensor], rows: int, cols: int, index: int, name: str):
    """Pointers and type of a tensor kept for the backward pass."""
    if t is None:
        return None, None, DB_BF16
    if t.dtype == _E4M3:
        if scale is None:
            raise ValueError(f"{name} in 8 bits needs its scale")
        return (_whole(t, (rows, cols), _E4M3, index, name),
                _whole(scale, (rows, checkpoint_scales(cols)), _E8M0, index, name + "'s scale"), DB_E4M3)
    return _whole(t, (rows, cols), _BF16, index, name), None, DB_BF16


def _grad_code(*tensors: Optional[torch.Tensor]):
    """The common type of the wanted weight gradients and its code."""
    dtype = None
    for t in tensors:
        if t is not None:
            if dtype is not None and t.dtype != dtype:
                raise TypeError("weight gradients must have one type")
            dtype = t.dtype
    return (_BF16, DB_BF16) if dtype is None else (dtype, _dtype_code(dtype))


def _scratch(t: torch.Tensor, index: int):
    """Pointer and size of a workspace: contiguous, so that its elements are the memory behind its pointer."""
    if t.get_device() != index:
        _elsewhere(t, index, "workspace")
    if not t.is_contiguous():
        raise TypeError("workspace must be a contiguous CUDA tensor")
    return t.data_ptr(), t.numel() * t.element_size()


def _launch(index: int, stream: Optional[torch.cuda.Stream], fn, *args) -> None:
    handle = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream
    if torch._C._cuda_getDevice() == index:
        status = fn(*args, handle)
    else:
        with torch.cuda.device(index):
            status = fn(*args, handle)
    if status:
        _check(status)


def _activation(name: str) -> int:
    try:
        return DB_ACTIVATIONS[name]
    except KeyError:
        raise ValueError(f"activation must be one of {sorted(DB_ACTIVATIONS)}") from None


def checkpoint_scales(n: int) -> int:
    """Scales of a row of n values of an 8-bit checkpoint."""
    return -(-int(n) // DB_CHECKPOINT_GROUP)


def linear_workspace_bytes(rows: int, n_in: int, n_out: int, aligned: bool = True) -> int:
    return int(lib().db_linear_workspace_bytes(_size(int(rows), 63), _size(int(n_in)), _size(int(n_out)), bool(aligned)))


def linear_grad_workspace_bytes(rows: int, n_in: int, n_out: int, aligned: bool = True) -> int:
    return int(lib().db_linear_grad_workspace_bytes(_size(int(rows), 63), _size(int(n_in)), _size(int(n_out)), bool(aligned)))


def gated_ffn_workspace_bytes(rows: int, width: int, hidden: int, aligned: bool = True) -> int:
    return int(lib().db_gated_ffn_workspace_bytes(_size(int(rows), 63), _size(int(width)), _size(int(hidden)), bool(aligned)))


def gated_ffn_grad_workspace_bytes(rows: int, width: int, hidden: int, aligned: bool = True) -> int:
    return int(lib().db_gated_ffn_grad_workspace_bytes(_size(int(rows), 63), _size(int(width)), _size(int(hidden)), bool(aligned)))


def linear(x: torch.Tensor, w: torch.Tensor, y: torch.Tensor, workspace: torch.Tensor, bias: Optional[torch.Tensor] = None,
           residual: Optional[torch.Tensor] = None, activation: str = "none", z: Optional[torch.Tensor] = None,
           z_scale: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_linear: y = activation(x w + bias) + residual, bfloat16.

    x [rows, n_in], y and residual [rows, n_out] may be slices of wider tensors (contiguous rows); w [n_in, n_out].
    z receives x w + bias for the backward pass: bfloat16, or float8_e4m3fn with z_scale [rows, checkpoint_scales(n_out)]
    (float8_e8m0fnu).  workspace: uint8, linear_workspace_bytes(...) bytes.
    """
    index = _device_index(x)
    rows, n_in = x.shape
    n_out = w.shape[-1]
    xp, x_pitch = _rows(x, rows, n_in, index, "x")
    rp, r_pitch = _rows(residual, rows, n_out, index, "residual")
    yp, y_pitch = _rows(y, rows, n_out, index, "y")
    zp, sp, zt = _kept(z, z_scale, rows, n_out, index, "z")
    _launch(index, stream, lib().db_linear, xp, x_pitch, _whole(w, (n_in, n_out), _BF16, index, "w"),
            _whole(bias, (n_out,), _BF16, index, "bias"), rp, r_pitch, _activation(activation), rows, _size(n_in), _size(n_out), yp, y_pitch,
            zp, sp, zt, *_scratch(workspace, index))


def linear_grad(dy: torch.Tensor, x: Optional[torch.Tensor], w: torch.Tensor, workspace: torch.Tensor,
                z: Optional[torch.Tensor] = None, z_scale: Optional[torch.Tensor] = None, activation: str = "none",
                dx: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                dx_addend: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_linear_grad: the wanted ones of dx (+ dx_addend), dw and dbias; z as db_linear kept it (needed with an
    activation).  dw and dbias are both float32 or both bfloat16; x is needed for dw.
    workspace: linear_grad_workspace_bytes(...) bytes."""
    index = _device_index(dy)
    n_in, n_out = w.shape
    rows = dy.shape[0]
    dyp, dy_pitch = _rows(dy, rows, n_out, index, "dy")
    xp, x_pitch = _rows(x, rows, n_in, index, "x")
    dxp, dx_pitch = _rows(dx, rows, n_in, index, "dx")
    ap, a_pitch = _rows(dx_addend, rows, n_in, index, "dx_addend")
    zp, sp, zt = _kept(z, z_scale, rows, n_out, index, "z")
    dtype, code = _grad_code(dw, dbias)
    _launch(index, stream, lib().db_linear_grad, dyp, dy_pitch, xp, x_pitch, _whole(w, (n_in, n_out), _BF16, index, "w"), zp, sp,
            zt, _activation(activation), rows, _size(n_in), _size(n_out), dxp, dx_pitch, ap, a_pitch,
            _whole(dw, (n_in, n_out), dtype, index, "dw"), _whole(dbias, (n_out,), dtype, index, "dbias"), code,
            *_scratch(workspace, index))


def gated_ffn(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, y: torch.Tensor,
              workspace: torch.Tensor, residual: Optional[torch.Tensor] = None, activation: str = "silu",
              gate: Optional[torch.Tensor] = None, up: Optional[torch.Tensor] = None,
              gate_scale: Optional[torch.Tensor] = None, up_scale: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_gated_ffn: y = (activation(x w_gate) * (x w_up)) w_down + residual, bfloat16.

    x, y, residual [rows, width] may be slices of wider tensors; w_gate, w_up [width, hidden], w_down [hidden, width].
    gate and up receive x w_gate and x w_up for the backward pass, both bfloat16 or both float8_e4m3fn with their scales
    [rows, checkpoint_scales(hidden)].  workspace: gated_ffn_workspace_bytes(...) bytes.
    """
    index = _device_index(x)
    rows, width = x.shape
    hidden = w_gate.shape[-1]
    xp, x_pitch = _rows(x, rows, width, index, "x")
    rp, r_pitch = _rows(residual, rows, width, index, "residual")
    yp, y_pitch = _rows(y, rows, width, index, "y")
    gp, gs, gt = _kept(gate, gate_scale, rows, hidden, index, "gate")
    upp, us, ut = _kept(up, up_scale, rows, hidden, index, "up")
    if gate is not None and up is not None and gt != ut:
        raise TypeError("gate and up must have one type")
    _launch(index, stream, lib().db_gated_ffn, xp, x_pitch, _whole(w_gate, (width, hidden), _BF16, index, "w_gate"),
            _whole(w_up, (width, hidden), _BF16, index, "w_up"), _whole(w_down, (hidden, width), _BF16, index, "w_down"), rp,
            r_pitch, _activation(activation), rows, _size(width), _size(hidden), yp, y_pitch, gp, upp, gs, us, gt,
            *_scratch(workspace, index))


def gated_ffn_grad(dy: torch.Tensor, x: Optional[torch.Tensor], w_gate: torch.Tensor, w_up: torch.Tensor,
                   w_down: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, workspace: torch.Tensor,
                   gate_scale: Optional[torch.Tensor] = None, up_scale: Optional[torch.Tensor] = None,
                   activation: str = "silu", dx: Optional[torch.Tensor] = None, dw_gate: Optional[torch.Tensor] = None,
                   dw_up: Optional[torch.Tensor] = None, dw_down: Optional[torch.Tensor] = None,
                   dx_addend: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_gated_ffn_grad: the wanted ones of dx (+ dx_addend), dw_gate, dw_up and dw_down; gate and up as db_gated_ffn kept
    them.  The weight gradients have one type, float32 or bfloat16; x is needed for dw_gate and dw_up.
    workspace: gated_ffn_grad_workspace_bytes(...) bytes."""
    index = _device_index(dy)
    width, hidden = w_gate.shape
    rows = dy.shape[0]
    dyp, dy_pitch = _rows(dy, rows, width, index, "dy")
    xp, x_pitch = _rows(x, rows, width, index, "x")
    dxp, dx_pitch = _rows(dx, rows, width, index, "dx")
    ap, a_pitch = _rows(dx_addend, rows, width, index, "dx_addend")
    gp, gs, gt = _kept(gate, gate_scale, rows, hidden, index, "gate")
    upp, us, ut = _kept(up, up_scale, rows, hidden, index, "up")
    if gt != ut:
        raise TypeError("gate and up must have one type")
    dtype, code = _grad_code(dw_gate, dw_up, dw_down)
    _launch(index, stream, lib().db_gated_ffn_grad, dyp, dy_pitch, xp, x_pitch,
            _whole(w_gate, (width, hidden), _BF16, index, "w_gate"), _whole(w_up, (width, hidden), _BF16, index, "w_up"),
            _whole(w_down, (hidden, width), _BF16, index, "w_down"), gp, upp, gs, us, gt, _activation(activation), rows,
            _size(width), _size(hidden), dxp, dx_pitch, ap, a_pitch, _whole(dw_gate, (width, hidden), dtype, index, "dw_gate"),
            _whole(dw_up, (width, hidden), dtype, index, "dw_up"), _whole(dw_down, (hidden, width), dtype, index, "dw_down"),
            code, *_scratch(workspace, index))


def layer_status(workspace: torch.Tensor) -> int:
    """The status word at the start of a layer call's workspace (0 = every internal wait completed)."""
    return int(workspace[:4].view(torch.int32).item())


def checkpoint_pack(x: torch.Tensor, codes: torch.Tensor, scale: torch.Tensor,
                    stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_checkpoint_pack: x [rows, cols] bfloat16 (rows contiguous) to codes [rows, cols] float8_e4m3fn and scale
    [rows, checkpoint_scales(cols)] float8_e8m0fnu."""
    index = _device_index(x)
    rows, cols = x.shape
    if codes.dtype != _E4M3:
        raise TypeError("codes must be float8_e4m3fn")
    xp, pitch = _rows(x, rows, cols, index, "x")
    cp, sp, _ = _kept(codes, scale, rows, cols, index, "codes")
    _launch(index, stream, lib().db_checkpoint_pack, xp, pitch, rows, _size(cols), cp, sp)


def checkpoint_unpack(codes: torch.Tensor, scale: torch.Tensor, x: torch.Tensor,
                      stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_checkpoint_unpack: the values that codes and scale stand for, rounded to bfloat16, into x."""
    index = _device_index(codes)
    rows, cols = codes.shape
    if codes.dtype != _E4M3:
        raise TypeError("codes must be float8_e4m3fn")
    xp, pitch = _rows(x, rows, cols, index, "x")
    cp, sp, _ = _kept(codes, scale, rows, cols, index, "codes")
    _launch(index, stream, lib().db_checkpoint_unpack, cp, sp, rows, _size(cols), xp, pitch)


def embedding(tokens: torch.Tensor, table: torch.Tensor, out: torch.Tensor, scale: float = 1.0,
              stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_embedding: out[t] = scale * table[tokens[t]]; tokens int32 (outside the table: zeros), table and out float32 or
    bfloat16, out's rows contiguous."""
    index = _device_index(tokens)
    vocab, width = table.shape
    rows = tokens.numel()
    op, pitch = _rows(out, rows, width, index, "out", out.dtype)
    _launch(index, stream, lib().db_embedding, _whole(tokens, tokens.shape, torch.int32, index, "tokens"),
            _whole(table, (vocab, width), table.dtype, index, "table"), _dtype_code(table.dtype), float(scale), rows, _size(vocab),
            _size(width), op, pitch, _dtype_code(out.dtype))


def embedding_grad_workspace_bytes(rows: int, vocab: int, width: int) -> int:
    return int(lib().db_embedding_grad_workspace_bytes(_size(int(rows), 63), _size(int(vocab)), _size(int(width))))


def embedding_grad(tokens: torch.Tensor, dy: torch.Tensor, dtable: torch.Tensor, workspace: torch.Tensor,
                   scale: float = 1.0, stream: Optional[torch.cuda.Stream] = None) -> None:
    """db_embedding_grad: dtable[v] = scale * sum of dy[t] with tokens[t] == v, every row written.  dy and dtable float32 or
    bfloat16; workspace: embedding_grad_workspace_bytes(rows, vocab, width) bytes."""
    index = _device_index(tokens)
    vocab, width = dtable.shape
    rows = tokens.numel()
    dp, pitch = _rows(dy, rows, width, index, "dy", dy.dtype)
    _launch(index, stream, lib().db_embedding_grad, _whole(tokens, tokens.shape, torch.int32, index, "tokens"), dp, pitch,
            _dtype_code(dy.dtype), float(scale), rows, _size(vocab), _size(width),
            _whole(dtable, (vocab, width), dtable.dtype, index, "dtable"), _dtype_code(dtable.dtype),
            *_scratch(workspace, index))
