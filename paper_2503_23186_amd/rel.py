"""Binding of include/cnnk_rel.h (argument marshalling only): dropout from a counter-based generator, and self-attention with
a learned relative position bias.  Every entry point runs inside libcnnk.so; there is no CPU fallback.

A training step's use: `rng` is a device tensor of two int64 (seed, step) that the forward and the backward calls of a step
read; cnnk_rng_advance moves its step on between training steps.  A bucket map (cnnk_rel_buckets_grid, or any [T][T] int32
tensor; numbers outside 0 .. buckets - 1 mask a pair) becomes a plan once, with make_plan."""
from __future__ import annotations
import ctypes as C
import functools
import torch
from .cnnk import lib, ptr, _check, F32, BF16  # noqa: F401

EXPORTS = ["cnnk_rng_advance", "cnnk_dropout_fwd", "cnnk_dropout_workspace_bytes", "cnnk_dropout_bwd", "cnnk_rel_buckets_grid",
           "cnnk_rel_plan_bytes", "cnnk_rel_plan_workspace_bytes", "cnnk_rel_plan", "cnnk_rel_attention_fwd",
           "cnnk_rel_attention_workspace_bytes", "cnnk_rel_attention_bwd"]


class DropoutDesc(C.Structure):
    _fields_ = [("rows", C.c_longlong), ("C", C.c_int), ("dtype", C.c_int), ("p", C.c_float), ("site", C.c_uint), ("span", C.c_int)]


class RelDesc(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("B", "T", "heads", "dh", "dtype", "buckets")] + [("p", C.c_float), ("site", C.c_uint)]


def _declare():
    vp, ci, sz, ull = C.c_void_p, C.c_int, C.c_size_t, C.c_ulonglong
    dd, rd = C.POINTER(DropoutDesc), C.POINTER(RelDesc)
    lib.cnnk_rng_advance.argtypes = [vp, ull, vp]
    lib.cnnk_dropout_fwd.argtypes = [dd, vp, vp, vp, vp, vp, vp]
    lib.cnnk_dropout_workspace_bytes.restype = sz
    lib.cnnk_dropout_workspace_bytes.argtypes = [dd]
    lib.cnnk_dropout_bwd.argtypes = [dd, vp, vp, vp, vp, vp, sz, vp]
    lib.cnnk_rel_buckets_grid.argtypes = [ci, ci, ci, vp, vp]
    lib.cnnk_rel_plan_bytes.restype = lib.cnnk_rel_plan_workspace_bytes.restype = sz
    lib.cnnk_rel_plan_bytes.argtypes = lib.cnnk_rel_plan_workspace_bytes.argtypes = [ci, ci]
    lib.cnnk_rel_plan.argtypes = [ci, ci, vp, vp, vp, sz, vp]
    lib.cnnk_rel_attention_fwd.argtypes = [rd] + [vp] * 8
    lib.cnnk_rel_attention_workspace_bytes.restype = sz
    lib.cnnk_rel_attention_workspace_bytes.argtypes = [rd]
    lib.cnnk_rel_attention_bwd.argtypes = [rd] + [vp] * 11 + [sz, vp]


_declare()


def cnnk_rng_advance(rng, by=1, stream=0):
    _check(lib.cnnk_rng_advance(ptr(rng), by, stream), "cnnk_rng_advance")


def dropout_desc(rows, Cc, dtype, p, site=0, span=0):
    return DropoutDesc(rows, Cc, dtype, p, site, span)


def cnnk_dropout_fwd(d, z, bias, res, rng, y, stream=0):
    _check(lib.cnnk_dropout_fwd(C.byref(d), ptr(z), ptr(bias), ptr(res), ptr(rng), ptr(y), stream), "cnnk_dropout_fwd")


def cnnk_dropout_workspace_bytes(d):
    return int(lib.cnnk_dropout_workspace_bytes(C.byref(d)))


def cnnk_dropout_bwd(d, dy, rng, dz, dbias=None, ws=None, ws_bytes=0, stream=0):
    _check(lib.cnnk_dropout_bwd(C.byref(d), ptr(dy), ptr(rng), ptr(dz), ptr(dbias), ptr(ws), ws_bytes, stream), "cnnk_dropout_bwd")


def grid_buckets(gh, gw, cls):
    """Buckets that cnnk_rel_buckets_grid uses."""
    return (2 * gh - 1) * (2 * gw - 1) + (3 if cls else 0)


def cnnk_rel_buckets_grid(gh, gw, cls, bucket, stream=0):
    _check(lib.cnnk_rel_buckets_grid(gh, gw, int(cls), ptr(bucket), stream), "cnnk_rel_buckets_grid")


def cnnk_rel_plan_bytes(T, buckets):
    return int(lib.cnnk_rel_plan_bytes(T, buckets))


def cnnk_rel_plan_workspace_bytes(T, buckets):
    return int(lib.cnnk_rel_plan_workspace_bytes(T, buckets))


def cnnk_rel_plan(T, buckets, bucket, plan, ws, ws_bytes, stream=0):
    _check(lib.cnnk_rel_plan(T, buckets, ptr(bucket), ptr(plan), ptr(ws), ws_bytes, stream), "cnnk_rel_plan")


def make_plan(bucket, buckets):
    """The plan of a [T][T] int32 device tensor, as a device tensor, made on the current stream of its device."""
    T = bucket.shape[0]
    if bucket.shape != (T, T) or bucket.dtype != torch.int32 or not bucket.is_cuda or not bucket.is_contiguous():
        raise ValueError("a bucket map is a contiguous [T][T] int32 tensor on a GPU")
    n = cnnk_rel_plan_bytes(T, buckets)
    if n == 0:
        raise ValueError("unsupported bucket map: %d tokens, %d buckets" % (T, buckets))
    with torch.cuda.device(bucket.device):
        plan = torch.empty(n, dtype=torch.uint8, device=bucket.device)
        ws = torch.empty(cnnk_rel_plan_workspace_bytes(T, buckets), dtype=torch.uint8, device=bucket.device)
        cnnk_rel_plan(T, buckets, bucket, plan, ws, ws.numel(), torch.cuda.current_stream().cuda_stream)
    return plan


def rel_desc(B, T, heads, dh, dtype, buckets=0, p=0.0, site=0):
    return RelDesc(B, T, heads, dh, dtype, buckets, p, site)


_plan_bytes = functools.lru_cache(4096)(cnnk_rel_plan_bytes)


def _plan(d, plan):
    """ptr() of a plan, which has to have the bytes that the call reads: a kernel cannot tell."""
    if plan is None or isinstance(plan, int):
        return plan
    if plan.nbytes < _plan_bytes(d.T, d.buckets):
        raise ValueError("the plan is too small for %d tokens and %d buckets" % (d.T, d.buckets))
    return plan.data_ptr()


def cnnk_rel_attention_fwd(d, qkv, table, plan, lens, rng, o, stats=None, stream=0):
    _check(lib.cnnk_rel_attention_fwd(C.byref(d), ptr(qkv), ptr(table), _plan(d, plan), ptr(lens), ptr(rng), ptr(o), ptr(stats), stream), "cnnk_rel_attention_fwd")


def cnnk_rel_attention_workspace_bytes(d):
    return int(lib.cnnk_rel_attention_workspace_bytes(C.byref(d)))


def cnnk_rel_attention_bwd(d, qkv, o, d_o, table, plan, lens, rng, stats, dqkv, dtable, ws, ws_bytes, stream=0):
    _check(lib.cnnk_rel_attention_bwd(C.byref(d), ptr(qkv), ptr(o), ptr(d_o), ptr(table), _plan(d, plan), ptr(lens),
                                      ptr(rng), ptr(stats), ptr(dqkv), ptr(dtable), ptr(ws), ws_bytes, stream),
           "cnnk_rel_attention_bwd")
