"""Thin Python binding of the C boundary declared in ``include/redist.h``.

Argument marshalling only: every step of a redistribution runs in the CUDA library.  PyTorch is
used for device memory and streams, nothing else.  There is no CPU fallback: if the library has
not been built, loading fails with an error that says how to build it.

A distributed type is ``(global_shape, axes)`` -- or any object with ``global_shape`` and ``axes``
attributes -- where ``axes[k]`` lists the mesh axes (indices into ``mesh_shape``) that partition
dimension ``k``, minor-to-major (Section 2.1 of the paper).
"""
from __future__ import annotations

import array
import contextlib
import ctypes
import json
import os
import struct
from typing import List, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("REDIST_LIB") or os.path.join(HERE, "libredist_b200.so")

FUSE_ADJACENT, FUSE_NONE, FUSE_ALL, NAIVE = 0, 1, 2, 3
NO_OVERPARTITION = 16
COST_PERMUTE = 32
NO_CACHE = 64
MAX_RANK = 8
STATIC_SCRATCH_BYTES = 8 << 20

STEP_KINDS = ("dynslice", "alltoall", "allgather", "allpermute", "copy")
KERNELS = ("dynslice", "alltoall", "allgather", "allpermute", "copy", "fused", "naive_gather", "naive_slice")

EXPORTS = (
    "redist_plan", "redist_plan_destroy", "redist_execute", "redist_execute_host", "redist_execute_static",
    "redist_bind", "redist_bound_execute", "redist_bound_destroy",
    "redist_plan_cache_stats", "redist_plan_cache_clear",
    "redist_tuning_set", "redist_tuning_get", "redist_tuning_reset", "redist_debug_bounds_report",
    "redist_plan_gpu_split",
    "redist_plan_num_devices", "redist_plan_rank", "redist_plan_local_elems", "redist_plan_scratch_bytes",
    "redist_plan_scratch_bytes_per_device", "redist_plan_staging_bytes", "redist_plan_alignment",
    "redist_plan_height", "redist_plan_cost", "redist_plan_num_steps", "redist_plan_num_launches",
    "redist_plan_step_info", "redist_plan_launch_info", "redist_plan_describe", "redist_base_offsets",
    "redist_status_string", "redist_last_cuda_error", "redist_bulk_timeouts",
    "redist_linear_scratch_bytes", "redist_linear_forward", "redist_linear_backward",
    "redist_layer_norm_forward", "redist_layer_norm_scratch_bytes", "redist_layer_norm_backward",
    "redist_orthogonalize_scratch_bytes", "redist_orthogonalize", "redist_product_timeouts",
    "redist_route_scratch_bytes", "redist_route_forward", "redist_route_backward",
    "redist_dispatch_forward", "redist_dispatch_backward", "redist_combine_forward", "redist_combine_backward",
    "redist_experts_scratch_bytes", "redist_experts_forward", "redist_experts_backward",
    "redist_clip_scratch_bytes", "redist_clip",
)

ACTIVATIONS = ("none", "relu", "gelu", "silu")


class RedistError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        self.status = int(status)
        msg = _status_string(status)
        super().__init__(f"{what}: {msg} (status {status})" if what else f"{msg} (status {status})")


class _Type(ctypes.Structure):
    _fields_ = [("rank", ctypes.c_int32), ("global_shape", ctypes.POINTER(ctypes.c_int64)),
                ("axes_off", ctypes.POINTER(ctypes.c_int32)), ("axes", ctypes.POINTER(ctypes.c_int32))]


class StepInfo(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("dim_i", ctypes.c_int32), ("dim_j", ctypes.c_int32),
                ("factor", ctypes.c_int64), ("local_before", ctypes.c_int64 * MAX_RANK),
                ("local_after", ctypes.c_int64 * MAX_RANK), ("cost", ctypes.c_int64),
                ("localsize_after", ctypes.c_int64)]


class LaunchInfo(ctypes.Structure):
    _fields_ = [("first_step", ctypes.c_int32), ("n_steps", ctypes.c_int32), ("kernel", ctypes.c_int32),
                ("vector_bytes", ctypes.c_int32), ("run_bytes", ctypes.c_int64), ("bytes_read", ctypes.c_int64),
                ("bytes_written", ctypes.c_int64), ("n_items", ctypes.c_int64), ("fanout", ctypes.c_int32),
                ("variant", ctypes.c_int32)]


class _Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("row_stride", ctypes.c_int64), ("col_stride", ctypes.c_int64)]


class _Linear(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("in_features", ctypes.c_int64), ("out_features", ctypes.c_int64),
                ("type", ctypes.c_int32), ("bias_type", ctypes.c_int32), ("activation", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("x", _Matrix), ("w", _Matrix), ("residual", _Matrix), ("out", _Matrix),
                ("pre", _Matrix), ("bias", ctypes.c_void_p)]


class _LinearGrads(ctypes.Structure):
    _fields_ = [("dy", _Matrix), ("dx", _Matrix), ("dw", _Matrix), ("dbias", ctypes.c_void_p)]


class _LayerNorm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("type", ctypes.c_int32),
                ("weight_type", ctypes.c_int32), ("eps", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("x", _Matrix), ("y", _Matrix), ("gamma", ctypes.c_void_p), ("beta", ctypes.c_void_p),
                ("mean", ctypes.c_void_p), ("rstd", ctypes.c_void_p)]


class _LayerNormGrads(ctypes.Structure):
    _fields_ = [("dy", _Matrix), ("dx", _Matrix), ("dgamma", ctypes.c_void_p), ("dbeta", ctypes.c_void_p)]


class _Orthogonal(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("type", ctypes.c_int32), ("steps", ctypes.c_int32), ("eps", ctypes.c_double),
                ("scale", ctypes.c_float), ("reserved", ctypes.c_int32), ("x", _Matrix), ("out", _Matrix),
                ("x_batch_stride", ctypes.c_int64), ("out_batch_stride", ctypes.c_int64),
                ("coefficients", ctypes.c_void_p)]


class _Route(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("experts", ctypes.c_int32), ("chosen", ctypes.c_int32),
                ("type", ctypes.c_int32), ("normalize", ctypes.c_int32), ("logits", _Matrix),
                ("weights", ctypes.c_void_p), ("choice", ctypes.c_void_p), ("position", ctypes.c_void_p),
                ("offsets", ctypes.c_void_p)]


class _Move(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("type", ctypes.c_int32), ("chosen", ctypes.c_int32), ("token", _Matrix), ("row", _Matrix),
                ("residual", _Matrix), ("drow", _Matrix), ("position", ctypes.c_void_p),
                ("weights", ctypes.c_void_p), ("dweights", ctypes.c_void_p)]


class _Experts(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("in_features", ctypes.c_int64), ("out_features", ctypes.c_int64),
                ("experts", ctypes.c_int32), ("type", ctypes.c_int32), ("bias_type", ctypes.c_int32),
                ("activation", ctypes.c_int32), ("x", _Matrix), ("w", _Matrix), ("out", _Matrix), ("pre", _Matrix),
                ("w_stride", ctypes.c_int64), ("bias_stride", ctypes.c_int64), ("bias", ctypes.c_void_p),
                ("offsets", ctypes.c_void_p)]


class _ExpertsGrads(ctypes.Structure):
    _fields_ = [("dy", _Matrix), ("dx", _Matrix), ("dw", _Matrix), ("dw_stride", ctypes.c_int64),
                ("dbias", ctypes.c_void_p)]


class _Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("out", ctypes.c_void_p), ("elements", ctypes.c_int64),
                ("type", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class _Clip(ctypes.Structure):
    _fields_ = [("tensors", ctypes.POINTER(_Tensor)), ("count", ctypes.c_int64), ("max_norm", ctypes.c_float),
                ("eps", ctypes.c_float), ("norm", ctypes.c_void_p)]


_lib = None


def load() -> ctypes.CDLL:
    """Load ``libredist_b200.so``; raise if it has not been built (no fallback of any kind)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2112_01075_b200.build` "
            "(needs nvcc; cross-compiles for sm_100a without a GPU)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.redist_plan.argtypes = [i32, ctypes.POINTER(i64), ctypes.POINTER(_Type), ctypes.POINTER(_Type), i32,
                                ctypes.c_uint32, ctypes.POINTER(vp)]
    lib.redist_plan.restype = i32
    lib.redist_plan_destroy.argtypes = [vp]
    lib.redist_plan_destroy.restype = None
    lib.redist_execute.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), vp, sz, vp]
    lib.redist_execute.restype = i32
    lib.redist_execute_static.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), vp]
    lib.redist_execute_static.restype = i32
    lib.redist_execute_host.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), vp, sz, vp, sz, vp, sz, vp]
    lib.redist_execute_host.restype = i32
    for name, res in (("redist_plan_num_devices", i32), ("redist_plan_rank", i32),
                      ("redist_plan_scratch_bytes", sz), ("redist_plan_scratch_bytes_per_device", sz),
                      ("redist_plan_alignment", i32), ("redist_plan_height", i64), ("redist_plan_cost", i64),
                      ("redist_plan_num_steps", i32), ("redist_plan_num_launches", i32)):
        getattr(lib, name).argtypes = [vp]
        getattr(lib, name).restype = res
    lib.redist_plan_local_elems.argtypes = [vp, i32]
    lib.redist_plan_local_elems.restype = i64
    lib.redist_plan_staging_bytes.argtypes = [vp, i32]
    lib.redist_plan_staging_bytes.restype = sz
    lib.redist_plan_step_info.argtypes = [vp, i32, ctypes.POINTER(StepInfo)]
    lib.redist_plan_step_info.restype = i32
    lib.redist_plan_launch_info.argtypes = [vp, i32, ctypes.POINTER(LaunchInfo)]
    lib.redist_plan_launch_info.restype = i32
    lib.redist_plan_describe.argtypes = [vp, ctypes.c_char_p, sz]
    lib.redist_plan_describe.restype = sz
    lib.redist_base_offsets.argtypes = [i32, ctypes.POINTER(i64), ctypes.POINTER(_Type), ctypes.POINTER(i64),
                                        ctypes.POINTER(i64)]
    lib.redist_base_offsets.restype = i32
    lib.redist_status_string.argtypes = [i32]
    lib.redist_status_string.restype = ctypes.c_char_p
    lib.redist_last_cuda_error.argtypes = []
    lib.redist_last_cuda_error.restype = i32
    lib.redist_bulk_timeouts.argtypes = []
    lib.redist_bulk_timeouts.restype = i64
    lib.redist_bind.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), vp, sz, ctypes.POINTER(vp)]
    lib.redist_bind.restype = i32
    lib.redist_bound_execute.argtypes = [vp, vp]
    lib.redist_bound_execute.restype = i32
    lib.redist_bound_destroy.argtypes = [vp]
    lib.redist_bound_destroy.restype = None
    lib.redist_plan_cache_stats.argtypes = [ctypes.POINTER(i64)] * 3
    lib.redist_plan_cache_stats.restype = None
    lib.redist_plan_cache_clear.argtypes = []
    lib.redist_plan_cache_clear.restype = None
    lib.redist_tuning_set.argtypes = [ctypes.c_char_p, i64]
    lib.redist_tuning_set.restype = i32
    lib.redist_tuning_get.argtypes = [ctypes.c_char_p, ctypes.POINTER(i64)]
    lib.redist_tuning_get.restype = i32
    lib.redist_tuning_reset.argtypes = []
    lib.redist_tuning_reset.restype = None
    lib.redist_plan_gpu_split.argtypes = [vp, i32, i32, ctypes.POINTER(i64)]
    lib.redist_plan_gpu_split.restype = i32
    lib.redist_linear_scratch_bytes.argtypes = [ctypes.POINTER(_Linear), ctypes.POINTER(_LinearGrads)]
    lib.redist_linear_scratch_bytes.restype = sz
    lib.redist_linear_forward.argtypes = [ctypes.POINTER(_Linear), vp, sz, vp]
    lib.redist_linear_forward.restype = i32
    lib.redist_linear_backward.argtypes = [ctypes.POINTER(_Linear), ctypes.POINTER(_LinearGrads), vp, sz, vp]
    lib.redist_linear_backward.restype = i32
    lib.redist_layer_norm_forward.argtypes = [ctypes.POINTER(_LayerNorm), vp]
    lib.redist_layer_norm_forward.restype = i32
    lib.redist_layer_norm_scratch_bytes.argtypes = [ctypes.POINTER(_LayerNorm), ctypes.POINTER(_LayerNormGrads)]
    lib.redist_layer_norm_scratch_bytes.restype = sz
    lib.redist_layer_norm_backward.argtypes = [ctypes.POINTER(_LayerNorm), ctypes.POINTER(_LayerNormGrads), vp, sz, vp]
    lib.redist_layer_norm_backward.restype = i32
    lib.redist_orthogonalize_scratch_bytes.argtypes = [ctypes.POINTER(_Orthogonal)]
    lib.redist_orthogonalize_scratch_bytes.restype = sz
    lib.redist_orthogonalize.argtypes = [ctypes.POINTER(_Orthogonal), vp, sz, vp]
    lib.redist_orthogonalize.restype = i32
    for name, blocks, scratch in (("route_forward", (_Route,), True), ("experts_forward", (_Experts,), True),
                                  ("experts_backward", (_Experts, _ExpertsGrads), True), ("clip", (_Clip,), True),
                                  ("dispatch_forward", (_Move,), False), ("dispatch_backward", (_Move,), False),
                                  ("combine_forward", (_Move,), False), ("combine_backward", (_Move,), False)):
        fn = getattr(lib, "redist_" + name)
        fn.argtypes, fn.restype = [ctypes.POINTER(b) for b in blocks] + ([vp, sz] if scratch else []) + [vp], i32
    lib.redist_route_backward.argtypes = [ctypes.POINTER(_Route), vp, ctypes.POINTER(_Matrix), vp]
    lib.redist_route_backward.restype = i32
    for name, blocks in (("route", (_Route,)), ("experts", (_Experts, _ExpertsGrads)), ("clip", (_Clip,))):
        fn = getattr(lib, f"redist_{name}_scratch_bytes")
        fn.argtypes, fn.restype = [ctypes.POINTER(b) for b in blocks], sz
    lib.redist_product_timeouts.argtypes = []
    lib.redist_product_timeouts.restype = i64
    lib.redist_debug_bounds_report.argtypes = [ctypes.POINTER(i64)]
    lib.redist_debug_bounds_report.restype = i32
    _lib = lib
    return lib


def _status_string(status: int) -> str:
    try:
        return load().redist_status_string(int(status)).decode()
    except Exception:
        return "?"


def _split(t):
    if hasattr(t, "global_shape"):
        return tuple(t.global_shape), tuple(tuple(a) for a in t.axes)
    return tuple(t[0]), tuple(tuple(a) for a in t[1])


class _CType:
    """Keeps the ctypes arrays of a redist_type alive."""

    def __init__(self, t):
        gshape, axes = _split(t)
        off, flat = [0], []
        for ax in axes:
            flat.extend(int(a) for a in ax)
            off.append(len(flat))
        self.shape = (ctypes.c_int64 * max(1, len(gshape)))(*[int(s) for s in gshape])
        self.off = (ctypes.c_int32 * len(off))(*off)
        self.flat = (ctypes.c_int32 * max(1, len(flat)))(*flat)
        self.struct = _Type(len(gshape), self.shape, self.off, self.flat)


def _mesh(mesh_shape):
    return (ctypes.c_int64 * max(1, len(mesh_shape)))(*[int(k) for k in mesh_shape])


def redist_base_offsets(mesh_shape: Sequence[int], dtype):
    """``(tile_shape, offsets)`` with ``offsets[d][k]`` the base offset of device ``d`` in dim ``k``."""
    lib = load()
    ct = _CType(dtype)
    rank = ct.struct.rank
    n = 1
    for k in mesh_shape:
        n *= int(k)
    tile = (ctypes.c_int64 * max(1, rank))()
    off = (ctypes.c_int64 * max(1, n * rank))()
    rc = lib.redist_base_offsets(len(mesh_shape), _mesh(mesh_shape), ctypes.byref(ct.struct), tile, off)
    if rc:
        raise RedistError(rc, "redist_base_offsets")
    return tuple(tile[:rank]), [tuple(off[d * rank:(d + 1) * rank]) for d in range(n)]


class Plan:
    """A synthesized redistribution (``redist_plan``).  Immutable; free with ``close()`` or GC."""

    def __init__(self, mesh_shape: Sequence[int], src, dst, elem_bytes: int, flags: int = FUSE_ADJACENT):
        lib = load()
        self._lib = lib
        self._h = ctypes.c_void_p()
        s, d = _CType(src), _CType(dst)
        rc = lib.redist_plan(len(mesh_shape), _mesh(mesh_shape), ctypes.byref(s.struct), ctypes.byref(d.struct),
                             int(elem_bytes), int(flags), ctypes.byref(self._h))
        if rc:
            self._h = None
            raise RedistError(rc, "redist_plan")
        self.mesh_shape = tuple(int(k) for k in mesh_shape)
        self.src, self.dst = _split(src), _split(dst)
        self.elem_bytes = int(elem_bytes)
        self.flags = int(flags)

    def close(self):
        if getattr(self, "_h", None):
            self._lib.redist_plan_destroy(self._h)
            self._h = None

    __del__ = close

    # ---- queries
    @property
    def n_devices(self) -> int:
        return self._lib.redist_plan_num_devices(self._h)

    @property
    def scratch_bytes(self) -> int:
        return self._lib.redist_plan_scratch_bytes(self._h)

    @property
    def scratch_bytes_per_device(self) -> int:
        return self._lib.redist_plan_scratch_bytes_per_device(self._h)

    @property
    def alignment(self) -> int:
        return self._lib.redist_plan_alignment(self._h)

    @property
    def height(self) -> int:
        return self._lib.redist_plan_height(self._h)

    @property
    def cost(self) -> int:
        return self._lib.redist_plan_cost(self._h)

    @property
    def num_steps(self) -> int:
        return self._lib.redist_plan_num_steps(self._h)

    @property
    def num_launches(self) -> int:
        return self._lib.redist_plan_num_launches(self._h)

    def local_elems(self, which: int) -> int:
        return self._lib.redist_plan_local_elems(self._h, which)

    def staging_bytes(self, which: int) -> int:
        return self._lib.redist_plan_staging_bytes(self._h, which)

    def step_info(self, step: int) -> StepInfo:
        out = StepInfo()
        rc = self._lib.redist_plan_step_info(self._h, step, ctypes.byref(out))
        if rc:
            raise RedistError(rc, "redist_plan_step_info")
        return out

    def launch_info(self, launch: int) -> LaunchInfo:
        out = LaunchInfo()
        rc = self._lib.redist_plan_launch_info(self._h, launch, ctypes.byref(out))
        if rc:
            raise RedistError(rc, "redist_plan_launch_info")
        return out

    def step_kinds(self) -> List[str]:
        return [STEP_KINDS[self.step_info(s).kind] for s in range(self.num_steps)]

    def launch_kernels(self) -> List[str]:
        return [KERNELS[self.launch_info(s).kernel] for s in range(self.num_launches)]

    def bytes_moved(self):
        """(read, written) HBM bytes summed over the launches."""
        infos = [self.launch_info(q) for q in range(self.num_launches)]
        return sum(i.bytes_read for i in infos), sum(i.bytes_written for i in infos)

    def gpu_split(self, n_gpus: int, launch: int):
        """``redist_plan_gpu_split``: ``m[s][t]`` = bytes GPU ``s`` would read locally and write to GPU ``t``
        if the virtual devices were spread over ``n_gpus`` GPUs by a prefix of the mesh axes."""
        out = (ctypes.c_int64 * (n_gpus * n_gpus))()
        rc = self._lib.redist_plan_gpu_split(self._h, n_gpus, launch, out)
        if rc:
            raise RedistError(rc, "redist_plan_gpu_split")
        return [[int(out[s * n_gpus + t]) for t in range(n_gpus)] for s in range(n_gpus)]

    def describe(self) -> dict:
        n = self._lib.redist_plan_describe(self._h, None, 0)
        buf = ctypes.create_string_buffer(n + 1)
        self._lib.redist_plan_describe(self._h, buf, n + 1)
        return json.loads(buf.value.decode())

    def pretty(self, axis_names: Optional[Sequence[str]] = None) -> str:
        """The synthesized sequence in the paper's notation, one collective per line, over the
        prime-factor mesh (axis ``x`` of size 4 appears as ``x.0, x.1``), followed by the launches."""
        d = self.describe()
        names = list(axis_names) if axis_names else [f"a{i}" for i in range(len(d["mesh_shape"]))]
        count: dict = {}
        pnames = []
        for p in d["primes"]:
            k = count.get(p["parent"], 0)
            count[p["parent"]] = k + 1
            pnames.append(f"{names[p['parent']]}.{k}")
        multi = {par for par, c in count.items() if c > 1}
        pnames = [n if d["primes"][i]["parent"] in multi else n.split(".")[0] for i, n in enumerate(pnames)]
        sizes = [p["size"] for p in d["primes"]]

        def fmt(axes):
            parts = []
            for s_k, ax in zip(d["global_shape"], axes):
                if not ax:
                    parts.append(str(s_k))
                    continue
                k = 1
                for a in ax:
                    k *= sizes[a]
                parts.append(f"{s_k // k}{{{','.join(pnames[a] for a in ax)}}}{s_k}")
            return "[" + ", ".join(parts) + "]"

        lines = [fmt(d["src_axes"])]
        for st in d["steps"]:
            label = st["kind"]
            if st["kind"] == "alltoall":
                label += f"({st['i']},{st['j']})"
            elif st["kind"] in ("allgather", "dynslice"):
                label += f"({st['i']})"
            if st["acting"]:
                label += "{" + ",".join(pnames[a] for a in st["acting"]) + "}"
            lines.append(f"  --{label}, cost {st['cost']}--> {fmt(st['post_axes'])}")
        for L in d["launches"]:
            g = L["geometry"]
            how = "ragged rows, TMA bulk loads" if g["bulk"] == 2 else "TMA bulk copies" if g["bulk"] else ("rows", "chunks", "units", "gather walk", "zip through shared memory", "super-boxes through shared memory")[g["mode"]]
            lines.append(f"  launch {L['kernel']}: steps {L['first_step']}..{L['first_step'] + L['n_steps'] - 1}, "
                         f"{L['from']} -> {L['to']}, runs of {L['run_bytes']} B, {g['n_items']} items, {how}")
        lines.append(f"  cost {d['cost']}, height {d['height']} <= max(localsize) "
                     f"{max(d['local_src'], d['local_dst'])}, scratch per device {d['scratch_per_device']} B")
        return "\n".join(lines)

    # ---- execution
    def execute_ptrs(self, src_ptrs: Sequence[int], dst_ptrs: Sequence[int], scratch_ptr: int = 0,
                     scratch_bytes: int = 0, stream: int = 0) -> None:
        """``redist_execute`` on raw device addresses."""
        n = len(src_ptrs)
        s = (ctypes.c_void_p * n)(*src_ptrs)
        d = (ctypes.c_void_p * len(dst_ptrs))(*dst_ptrs)
        rc = self._lib.redist_execute(self._h, s, d, ctypes.c_void_p(scratch_ptr or None), scratch_bytes,
                                      ctypes.c_void_p(stream or None))
        if rc:
            raise RedistError(rc, "redist_execute")

    def bind(self, src_ptrs: Sequence[int], dst_ptrs: Sequence[int], scratch_ptr: int = 0,
             scratch_bytes: int = 0):
        """``redist_bind``: validate the buffers and prepare every launch once; the returned callable runs
        ``redist_bound_execute`` on a stream (``call(stream_ptr)``) -- the kernel launches and nothing else.
        The buffers must stay alive and in place as long as the callable is used."""
        if len(src_ptrs) != self.n_devices or len(dst_ptrs) != self.n_devices:
            raise RedistError(1, "one tile per virtual device is required")
        s = (ctypes.c_void_p * len(src_ptrs))(*src_ptrs)
        d = (ctypes.c_void_p * len(dst_ptrs))(*dst_ptrs)
        h = ctypes.c_void_p()
        rc = self._lib.redist_bind(self._h, s, d, ctypes.c_void_p(scratch_ptr or None), scratch_bytes, ctypes.byref(h))
        if rc:
            raise RedistError(rc, "redist_bind")
        return _Bound(self, h)

    def _check_tiles(self, src_shards, dst_shards, cuda: bool = True) -> None:
        """What the C entry points cannot know: one tile per virtual device, each a contiguous tensor in
        the right memory holding exactly localsize*elem_bytes bytes."""
        if len(src_shards) != self.n_devices or len(dst_shards) != self.n_devices:
            raise RedistError(1, "one tile per virtual device is required")
        sb, db = self.local_elems(0) * self.elem_bytes, self.local_elems(1) * self.elem_bytes
        for t, need in [(x, sb) for x in src_shards] + [(x, db) for x in dst_shards]:
            if t.is_cuda != cuda or not t.is_contiguous() or t.numel() * t.element_size() != need:
                raise RedistError(1, "tiles must be contiguous %s tensors of the local size" % ("CUDA" if cuda else "host"))

    def execute(self, src_shards, dst_shards, scratch=None, stream=None) -> None:
        """``redist_execute`` on lists of CUDA tensors (one per virtual device), asynchronous."""
        import torch

        self._check_tiles(src_shards, dst_shards)
        if stream is None:
            stream = torch.cuda.current_stream()
        sp = scratch.data_ptr() if scratch is not None else 0
        sn = scratch.numel() * scratch.element_size() if scratch is not None else 0
        self.execute_ptrs([t.data_ptr() for t in src_shards], [t.data_ptr() for t in dst_shards], sp, sn,
                          stream.cuda_stream)

    def execute_static(self, src_shards, dst_shards, stream=None) -> None:
        """``redist_execute_static``: like ``execute`` but the scratch of an unfused plan comes from
        the fixed array built into the library, for callers that cannot allocate device memory
        (plans needing more than ``STATIC_SCRATCH_BYTES`` are refused)."""
        import torch

        self._check_tiles(src_shards, dst_shards)
        if stream is None:
            stream = torch.cuda.current_stream()
        n = self.n_devices
        s = (ctypes.c_void_p * n)(*[t.data_ptr() for t in src_shards])
        d = (ctypes.c_void_p * n)(*[t.data_ptr() for t in dst_shards])
        rc = self._lib.redist_execute_static(self._h, s, d, ctypes.c_void_p(stream.cuda_stream or None))
        if rc:
            raise RedistError(rc, "redist_execute_static")

    def execute_host(self, src_host, dst_host, dev_src, dev_dst, scratch=None, stream=None) -> None:
        """``redist_execute_host``: host tiles in, host tiles out, staged through ``dev_src``/``dev_dst``."""
        import torch

        self._check_tiles(src_host, dst_host, cuda=False)
        if stream is None:
            stream = torch.cuda.current_stream()
        n = self.n_devices
        s = (ctypes.c_void_p * n)(*[t.data_ptr() for t in src_host])
        d = (ctypes.c_void_p * n)(*[t.data_ptr() for t in dst_host])
        sp = scratch.data_ptr() if scratch is not None else 0
        sn = scratch.numel() * scratch.element_size() if scratch is not None else 0
        rc = self._lib.redist_execute_host(self._h, s, d, ctypes.c_void_p(dev_src.data_ptr()),
                                           dev_src.numel() * dev_src.element_size(),
                                           ctypes.c_void_p(dev_dst.data_ptr()),
                                           dev_dst.numel() * dev_dst.element_size(), ctypes.c_void_p(sp or None), sn,
                                           ctypes.c_void_p(stream.cuda_stream or None))
        if rc:
            raise RedistError(rc, "redist_execute_host")

    def alloc_scratch(self, device="cuda"):
        import torch

        n = self.scratch_bytes
        return torch.empty(n, dtype=torch.uint8, device=device) if n else None


class _Bound:
    """A plan bound to one set of buffers (``redist_bind``); calling it launches the kernels on a stream."""

    def __init__(self, plan: Plan, handle):
        self._plan, self._h = plan, handle          # the plan object stays alive with its bound form
        self._fn, self._destroy = plan._lib.redist_bound_execute, plan._lib.redist_bound_destroy

    def __call__(self, stream_ptr: int = 0) -> None:
        rc = self._fn(self._h, stream_ptr or None)      # argtypes convert the integer; nothing is built per call
        if rc:
            raise RedistError(rc, "redist_bound_execute")

    def close(self):
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None

    __del__ = close


def tuning_set(name: str, value: int) -> None:
    """``redist_tuning_set``: change a tuning value for the plans created from now on."""
    rc = load().redist_tuning_set(name.encode(), int(value))
    if rc:
        raise RedistError(rc, f"redist_tuning_set({name!r}, {value})")


def tuning_get(name: str) -> int:
    out = ctypes.c_int64()
    rc = load().redist_tuning_get(name.encode(), ctypes.byref(out))
    if rc:
        raise RedistError(rc, f"redist_tuning_get({name!r})")
    return int(out.value)


def tuning_reset() -> None:
    load().redist_tuning_reset()


@contextlib.contextmanager
def tuning(**values):
    """``with tuning(bulk=0, gather=0): plan = Plan(...)`` -- plans created inside get these values."""
    try:
        for k, v in values.items():
            tuning_set(k, v)
        yield
    finally:
        tuning_reset()


def plan_cache_stats():
    """``(hits, misses, entries)`` of the plan cache."""
    h, m, e = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
    load().redist_plan_cache_stats(ctypes.byref(h), ctypes.byref(m), ctypes.byref(e))
    return int(h.value), int(m.value), int(e.value)


def plan_cache_clear() -> None:
    load().redist_plan_cache_clear()


def debug_bounds_report():
    """Checked build only: ``(violations, line, block, side, distance)`` since the last call."""
    out = (ctypes.c_int64 * 5)()
    rc = load().redist_debug_bounds_report(out)
    if rc:
        raise RedistError(rc, "redist_debug_bounds_report")
    return tuple(int(v) for v in out)


def redist_bulk_timeouts() -> int:
    """Work items whose bounded bulk-copy wait ran out on the current device (0 in a healthy run)."""
    return int(load().redist_bulk_timeouts())


def redist_plan(mesh_shape, src, dst, elem_bytes: int, flags: int = FUSE_ADJACENT) -> Plan:
    return Plan(mesh_shape, src, dst, elem_bytes, flags)


def redist_execute(plan: Plan, src_shards, dst_shards, scratch=None, stream=None) -> None:
    plan.execute(src_shards, dst_shards, scratch, stream)


def shard_global(G, mesh_shape, dtype) -> list:
    """Cut a global tensor ``G`` (any device) into the tiles the type prescribes, one contiguous
    tensor per virtual device, using the library's base offset map."""
    tile, offs = redist_base_offsets(mesh_shape, dtype)
    out = []
    for off in offs:
        t = G
        for k, (o, c) in enumerate(zip(off, tile)):
            t = t.narrow(k, int(o), int(c))
        out.append(t.contiguous())
    return out


# ---- operators on a device's tiles -------------------------------------------------------------------
#
# Tensors in, tensors out; outputs that are not given are allocated.  Everything runs asynchronously on
# ``stream`` (default: the current one); what a call allocates itself, scratch included, is allocated on
# that stream, so the caching allocator hands it on in stream order.  Tensors of another stream than their
# own need the usual care of the caller (wait_stream, record_stream).
#
# Autograd does not see the operators: results require no gradient, whatever the arguments do, and the gradients are
# calls of their own (:func:`linear_backward`, :func:`layer_norm_backward`), to be put into a
# ``torch.autograd.Function`` where a graph is wanted.  Tensors of the caller that a call writes get a new version, so that a
# graph which kept their old contents refuses to go on with the new ones.
#
# The smallest calls take less time on the GPU than a few dozen lines of Python: arguments go over as one
# packed block per call (the layout of the C structures), and scratch is asked for where it is needed.

_MATRIX = "Pqq"
_pack_linear = struct.Struct("3q4i" + _MATRIX * 5 + "P").pack
_pack_linear_grads = struct.Struct(_MATRIX * 3 + "P").pack
_pack_layer_norm = struct.Struct("2q2ifi" + _MATRIX * 2 + "4P").pack
_pack_layer_norm_grads = struct.Struct(_MATRIX * 2 + "2P").pack
_pack_orthogonal = struct.Struct("3q2idfi" + _MATRIX * 2 + "2qP").pack
_pack_route = struct.Struct("q4i" + _MATRIX + "4P").pack
_pack_matrix = struct.Struct(_MATRIX).pack
_pack_move = struct.Struct("3q2i" + _MATRIX * 4 + "3P").pack
_pack_experts = struct.Struct("3q4i" + _MATRIX * 4 + "2q2P").pack
_pack_experts_grads = struct.Struct(_MATRIX * 3 + "qP").pack
_pack_clip = struct.Struct("Pq2fP").pack
_ESCRATCH = 5

_ops = None


class _Operators:
    """torch, its type codes, and the entry points with the argument types of a packed block."""

    def __init__(self):
        import torch

        lib = load()
        self.torch, self.empty, self.strided = torch, torch.empty, torch.empty_strided
        self.written = torch.autograd.graph.increment_version
        self.codes = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
        self.u8, self.f32, self.bf16, self.i32 = torch.uint8, torch.float32, torch.bfloat16, torch.int32
        self.current_device = self.raw_stream = None
        if torch.cuda.is_available():
            torch.cuda.init()
            self.current_device, self.raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        for name, blocks, scratch in (("linear_forward", 1, True), ("linear_backward", 2, True), ("layer_norm_forward", 1, False),
                                      ("layer_norm_backward", 2, True), ("orthogonalize", 1, True), ("route_forward", 1, True),
                                      ("route_backward", 3, False), ("dispatch_forward", 1, False), ("dispatch_backward", 1, False),
                                      ("combine_forward", 1, False), ("combine_backward", 1, False), ("experts_forward", 1, True),
                                      ("experts_backward", 2, True), ("clip", 1, True)):
            fn = lib["redist_" + name]                       # an object of its own: the attribute keeps its types
            fn.argtypes, fn.restype = [vp] * blocks + ([vp, sz] if scratch else []) + [vp], ctypes.c_int32
            setattr(self, name, fn)
        for name, blocks in (("linear", 2), ("layer_norm", 2), ("orthogonalize", 1), ("route", 1), ("experts", 2), ("clip", 1)):
            fn = lib[f"redist_{name}_scratch_bytes"]
            fn.argtypes, fn.restype = [vp] * blocks, sz
            setattr(self, name + "_scratch_bytes", fn)

    def stream(self, device, given):
        """The stream a call on ``device`` runs on (an address)."""
        if device.type != "cuda" or self.current_device is None:
            raise RedistError(1, "CUDA tensors are required")
        index = device.index
        if index != self.current_device():
            raise RedistError(1, "tensors have to be on the current device")
        return given.cuda_stream if given is not None else self.raw_stream(index)

    def matrix(self, rows, cols, dtype, device):
        """An uninitialised row-major matrix (half the time of torch.empty)."""
        return self.strided((rows, cols), (cols, 1), dtype=dtype, device=device)

    def scratch(self, need, given, device):
        """(tensor, address, bytes) of the scratch of one call."""
        if not need:
            return None, None, 0
        if given is None:
            given = self.strided((need,), (1,), dtype=self.u8, device=device)
        elif given.device != device or not given.is_contiguous():
            raise RedistError(1, f"scratch has to be a contiguous tensor on {device}")
        return given, given.data_ptr(), given.numel() * given.element_size()


def _operators() -> _Operators:
    global _ops
    if _ops is None:
        _ops = _Operators()
    return _ops


def _allocating(stream):
    """A context in which torch allocates for ``stream``."""
    if stream is None:
        return contextlib.nullcontext()
    import torch
    return torch.cuda.stream(stream)


def _code(o, t, what: str) -> int:
    code = o.codes.get(t.dtype)
    if code is None:
        raise RedistError(1, f"{what} is bfloat16, float16 or float32, not {t.dtype}")
    return code


def _matrix(t, shape, dtype, device, what: str):
    """``t`` as the three fields of a redist_matrix, checked."""
    if t is None:
        return 0, 0, 0
    if t.shape != shape:
        raise RedistError(1, f"{what} has to be {shape[0]} x {shape[1]}, not {tuple(t.shape)}")
    if t.dtype is not dtype or t.device != device:
        raise RedistError(1, f"{what} has to be of {dtype} on {device}, not {t.dtype} on {t.device}")
    a, b = t.stride()
    return t.data_ptr(), a, b


def _vector(o, t, length: int, device, what: str, dtype=None):
    """Address and type code of a contiguous vector."""
    if t is None:
        return 0, 0
    if t.dim() != 1 or t.shape[0] != length or t.device != device or not t.is_contiguous():
        raise RedistError(1, f"{what} has to be a contiguous vector of {length} elements on {device}")
    if dtype is not None and t.dtype is not dtype:
        raise RedistError(1, f"{what} has to be of {dtype}")
    code = o.codes.get(t.dtype)
    return t.data_ptr(), code if code is not None else _code(o, t, what)


_ACTIVATION_CODES = {name: code for code, name in enumerate(ACTIVATIONS)}


def _activation(name: str) -> int:
    code = _ACTIVATION_CODES.get(name)
    if code is None:
        raise RedistError(1, f"activation is one of {ACTIVATIONS}, not {name!r}")
    return code


def _not_matrices(**tensors) -> None:
    for name, t in tensors.items():
        if t.dim() != 2:
            raise RedistError(1, f"{name} has to be a matrix, not of {t.dim()} dimensions")


def linear_forward(x, w, bias=None, residual=None, activation: str = "none", out=None, pre=None, scratch=None, stream=None):
    """``redist_linear_forward``: ``activation(x @ w.T + bias) + residual``, in one pass over the products.

    ``x`` (rows, in) and ``w`` (out, in), bfloat16 or float16, rows or columns contiguous; ``bias`` (out,) of any
    type; ``residual`` (rows, out); ``pre`` (rows, out), if given, receives ``x @ w.T + bias`` for the backward pass.
    Returns ``out`` (rows, out)."""
    if stream is not None:
        with _allocating(stream):
            return _linear_forward(x, w, bias, residual, activation, out, pre, scratch, stream)
    return _linear_forward(x, w, bias, residual, activation, out, pre, scratch, None)


def _linear_forward(x, w, bias, residual, activation, out, pre, scratch, stream):
    o = _ops or _operators()
    if x.dim() != 2 or w.dim() != 2:
        _not_matrices(x=x, w=w)
    rows, k = x.shape
    n = w.shape[0]
    device, dtype, shape = x.device, x.dtype, (rows, n)
    at = o.stream(device, stream)
    given = out is not None
    if not given:
        out = o.matrix(rows, n, dtype, device)
    b, bt = _vector(o, bias, n, device, "bias")
    op = _pack_linear(rows, k, n, _code(o, x, "x"), bt, _activation(activation), 0, x.data_ptr(), *x.stride(),
                      *_matrix(w, (n, k), dtype, device, "w"), *_matrix(residual, shape, dtype, device, "residual"),
                      *_matrix(out, shape, dtype, device, "out"), *_matrix(pre, shape, dtype, device, "pre"), b)
    rc = o.linear_forward(op, None, 0, at) if scratch is None else _ESCRATCH
    if rc == _ESCRATCH:                                      # operands off 16-byte boundaries: rare
        keep, sp, sn = o.scratch(o.linear_scratch_bytes(op, None), scratch, device)
        rc = o.linear_forward(op, sp, sn, at)
    if rc:
        raise RedistError(rc, "redist_linear_forward")
    if pre is not None or given:
        o.written([t for t in (pre, out) if t is not None])
    return out


def linear_backward(dy, x, w, pre=None, activation: str = "none", need=(True, True, True), dx=None, dw=None, dbias=None,
                    scratch=None, stream=None):
    """``redist_linear_backward``: ``(dx, dw, dbias)``, the gradients of :func:`linear_forward` (that of ``residual`` is
    ``dy`` itself).  ``need`` says which of the three are wanted; the others are None.  ``pre`` is what the forward pass
    kept (not needed without an activation).  dx and dw have the type of ``dy``, dbias is float32."""
    if stream is not None:
        with _allocating(stream):
            return _linear_backward(dy, x, w, pre, activation, need, dx, dw, dbias, scratch, stream)
    return _linear_backward(dy, x, w, pre, activation, need, dx, dw, dbias, scratch, None)


def _linear_backward(dy, x, w, pre, activation, need, dx, dw, dbias, scratch, stream):
    o = _ops or _operators()
    if dy.dim() != 2 or x.dim() != 2 or w.dim() != 2:
        _not_matrices(dy=dy, x=x, w=w)
    rows, n = dy.shape
    k = x.shape[1]
    device, dtype = dy.device, dy.dtype
    at = o.stream(device, stream)
    wide, tall, long = (rows, n), (rows, k), (n, k)
    given = [t for t, wanted in zip((dx, dw, dbias), need) if wanted and t is not None]
    if not need[0]:
        dx = None
    elif dx is None:
        dx = o.matrix(rows, k, dtype, device)
    if not need[1]:
        dw = None
    elif dw is None:
        dw = o.matrix(n, k, dtype, device)
    if not need[2]:
        dbias = None
    elif dbias is None:
        dbias = o.strided((n,), (1,), dtype=o.f32, device=device)
    op = _pack_linear(rows, k, n, _code(o, dy, "dy"), 0, _activation(activation), 0, *_matrix(x, tall, dtype, device, "x"),
                      *_matrix(w, long, dtype, device, "w"), 0, 0, 0, 0, 0, 0, *_matrix(pre, wide, dtype, device, "pre"), 0)
    g = _pack_linear_grads(dy.data_ptr(), *dy.stride(), *_matrix(dx, tall, dtype, device, "dx"),
                           *_matrix(dw, long, dtype, device, "dw"), _vector(o, dbias, n, device, "dbias", o.f32)[0])
    keep, sp, sn = o.scratch(o.linear_scratch_bytes(op, g), scratch, device)
    rc = o.linear_backward(op, g, sp, sn, at)
    if rc:
        raise RedistError(rc, "redist_linear_backward")
    if given:
        o.written(given)
    return dx, dw, dbias


def layer_norm_forward(x, gamma=None, beta=None, eps: float = 1e-5, out=None, stream=None):
    """``redist_layer_norm_forward``: ``(y, mean, rstd)``.  ``x`` (rows, cols) in bfloat16, float16 or float32 with
    contiguous rows; ``gamma`` and ``beta`` (cols,), both of one type; ``mean`` and ``rstd`` (rows,) in float32 are
    what the backward pass needs."""
    if stream is not None:
        with _allocating(stream):
            return _layer_norm_forward(x, gamma, beta, eps, out, stream)
    return _layer_norm_forward(x, gamma, beta, eps, out, None)


def _layer_norm_forward(x, gamma, beta, eps, out, stream):
    o = _ops or _operators()
    if x.dim() != 2:
        _not_matrices(x=x)
    shape, dtype, device = x.shape, x.dtype, x.device
    rows, cols = shape
    at = o.stream(device, stream)
    given = out is not None
    if not given:
        out = o.matrix(rows, cols, dtype, device)
    mean, rstd = o.matrix(2, rows, o.f32, device).unbind()
    g, gt = _vector(o, gamma, cols, device, "gamma")
    b, bt = _vector(o, beta, cols, device, "beta")
    if g and b and gt != bt:
        raise RedistError(1, "gamma and beta have to be of one type")
    op = _pack_layer_norm(rows, cols, _code(o, x, "x"), gt if g else bt, eps, 0, x.data_ptr(), *x.stride(),
                          *_matrix(out, shape, dtype, device, "out"), g, b, mean.data_ptr(), rstd.data_ptr())
    rc = o.layer_norm_forward(op, at)
    if rc:
        raise RedistError(rc, "redist_layer_norm_forward")
    if given:
        o.written(out)
    return out, mean, rstd


def layer_norm_backward(dy, x, gamma, mean, rstd, dx=None, scratch=None, stream=None):
    """``redist_layer_norm_backward``: ``(dx, dgamma, dbeta)``; the last two are float32.  ``mean`` and ``rstd`` are the
    forward pass's; ``gamma`` may be None."""
    if stream is not None:
        with _allocating(stream):
            return _layer_norm_backward(dy, x, gamma, mean, rstd, dx, scratch, stream)
    return _layer_norm_backward(dy, x, gamma, mean, rstd, dx, scratch, None)


def _layer_norm_backward(dy, x, gamma, mean, rstd, dx, scratch, stream):
    o = _ops or _operators()
    if dy.dim() != 2:
        _not_matrices(dy=dy)
    shape, dtype, device = dy.shape, dy.dtype, dy.device
    rows, cols = shape
    at = o.stream(device, stream)
    given = dx is not None
    if not given:
        dx = o.matrix(rows, cols, dtype, device)
    dgamma, dbeta = o.matrix(2, cols, o.f32, device).unbind()
    if mean is None or rstd is None:
        raise RedistError(1, "mean and rstd are required")
    g, gt = _vector(o, gamma, cols, device, "gamma")
    op = _pack_layer_norm(rows, cols, _code(o, dy, "dy"), gt, 0.0, 0, *_matrix(x, shape, dtype, device, "x"), 0, 0, 0, g, 0,
                          _vector(o, mean, rows, device, "mean", o.f32)[0], _vector(o, rstd, rows, device, "rstd", o.f32)[0])
    grads = _pack_layer_norm_grads(dy.data_ptr(), *dy.stride(), *_matrix(dx, shape, dtype, device, "dx"), dgamma.data_ptr(),
                                   dbeta.data_ptr())
    keep, sp, sn = o.scratch(o.layer_norm_scratch_bytes(op, grads), scratch, device)
    rc = o.layer_norm_backward(op, grads, sp, sn, at)
    if rc:
        raise RedistError(rc, "redist_layer_norm_backward")
    if given:
        o.written(dx)
    return dx, dgamma, dbeta


def orthogonalize(x, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7, scale: float = 1.0,
                  out=None, scratch=None, stream=None):
    """``redist_orthogonalize``: every matrix of ``x`` -- (rows, cols) or (batch, rows, cols), bfloat16, float16 or
    float32, rows contiguous -- after ``steps`` Newton-Schulz steps, times ``scale``, in bfloat16.  ``coefficients`` is
    one triple for all steps, or one triple per step."""
    if stream is not None:
        with _allocating(stream):
            return _orthogonalize(x, steps, coefficients, eps, scale, out, scratch, stream)
    return _orthogonalize(x, steps, coefficients, eps, scale, out, scratch, None)


def _orthogonalize(x, steps, coefficients, eps, scale, out, scratch, stream):
    o = _ops or _operators()
    if x.dim() not in (2, 3):
        raise RedistError(1, "x is a matrix or a stack of matrices")
    if not 1 <= steps <= 64:
        raise RedistError(1, "1 to 64 steps")
    flat = [float(v) for c in coefficients for v in (c if hasattr(c, "__len__") else (c,))]
    if len(flat) == 3:
        flat = flat * steps
    if len(flat) != 3 * steps:
        raise RedistError(1, "coefficients is one triple, or one per step")
    shape, device = x.shape, x.device
    at = o.stream(device, stream)
    code = _code(o, x, "x")
    given = out is not None
    if not given:
        out = o.empty(shape, dtype=o.bf16, device=device)
    elif out.shape != shape or out.dtype is not o.bf16 or out.device != device:
        raise RedistError(1, "out has to be x's shape in bfloat16")
    if x.numel() == 0:
        return out
    batch, xs, os = (shape[0], x.stride(), out.stride()) if len(shape) == 3 else (1, (0, *x.stride()), (0, *out.stride()))
    triples = (ctypes.c_float * len(flat))(*flat)
    op = _pack_orthogonal(batch, shape[-2], shape[-1], code, steps, eps, scale, 0, x.data_ptr(), xs[1], xs[2], out.data_ptr(), os[1],
                          os[2], xs[0], os[0], ctypes.addressof(triples))
    keep, sp, sn = o.scratch(o.orthogonalize_scratch_bytes(op), scratch, device)
    rc = o.orthogonalize(op, sp, sn, at)
    if rc:
        raise RedistError(rc, "redist_orthogonalize")
    if given:
        o.written(out)
    return out


# ---- a block of experts -------------------------------------------------------------------------------
#
# Nothing here asks the device for a size: a token has ``k`` places whatever the choice, ``tokens * k`` rows hold them in the
# order of the experts, and where an expert's rows begin (``offsets``) stays on the device.


def _table(o, t, shape, dtype, device, what: str) -> int:
    """Address of a contiguous tensor."""
    if t is None:
        raise RedistError(1, f"{what} is required")
    if t.shape != shape or t.dtype is not dtype or t.device != device or not t.is_contiguous():
        raise RedistError(1, f"{what} has to be a contiguous tensor of {tuple(shape)}, {dtype}, on {device}")
    return t.data_ptr()


def route_forward(logits, k: int, normalize: bool = True, scratch=None, stream=None):
    """``redist_route_forward``: ``(weights, choice, position, offsets)`` for the ``k`` experts of each token with the largest
    ``logits`` (tokens, experts) -- ties to the lower index, minus infinity never.

    ``weights`` (tokens, k) float32: softmax over the chosen experts, or, without ``normalize``, over all of them;
    ``choice`` (tokens, k) int32: the experts, -1 in places that stay empty; ``position`` (tokens, k) int32: the places'
    rows in the order of the experts (-1); ``offsets`` (experts + 1,) int32: where each expert's rows begin."""
    if stream is not None:
        with _allocating(stream):
            return _route_forward(logits, k, normalize, scratch, stream)
    return _route_forward(logits, k, normalize, scratch, None)


def _route_forward(logits, k, normalize, scratch, stream):
    o = _ops or _operators()
    if logits.dim() != 2:
        _not_matrices(logits=logits)
    tokens, experts = logits.shape
    if not 1 <= k <= experts:
        raise RedistError(1, f"1 to {experts} experts can be chosen, not {k}")
    device = logits.device
    at = o.stream(device, stream)
    weights = o.matrix(tokens, k, o.f32, device)
    choice, position = o.strided((2, tokens, k), (tokens * k, k, 1), dtype=o.i32, device=device).unbind()
    offsets = o.strided((experts + 1,), (1,), dtype=o.i32, device=device)
    op = _pack_route(tokens, experts, k, _code(o, logits, "logits"), 1 if normalize else 0, logits.data_ptr(), *logits.stride(),
                     weights.data_ptr(), choice.data_ptr(), position.data_ptr(), offsets.data_ptr())
    rc = o.route_forward(op, None, 0, at) if scratch is None else _ESCRATCH
    if rc == _ESCRATCH:                                      # many tokens
        keep, sp, sn = o.scratch(o.route_scratch_bytes(op), scratch, device)
        rc = o.route_forward(op, sp, sn, at)
    if rc:
        raise RedistError(rc, "redist_route_forward")
    return weights, choice, position, offsets


def route_backward(dweights, logits, weights, choice, normalize: bool = True, dlogits=None, stream=None):
    """``redist_route_backward``: ``dlogits`` (tokens, experts), of the type of ``logits``, from the gradient ``dweights``
    (tokens, k) float32 of the forward pass's ``weights``."""
    if stream is not None:
        with _allocating(stream):
            return _route_backward(dweights, logits, weights, choice, normalize, dlogits, stream)
    return _route_backward(dweights, logits, weights, choice, normalize, dlogits, None)


def _route_backward(dweights, logits, weights, choice, normalize, dlogits, stream):
    o = _ops or _operators()
    if logits.dim() != 2 or choice.dim() != 2:
        _not_matrices(logits=logits, choice=choice)
    shape, dtype, device = logits.shape, logits.dtype, logits.device
    tokens, experts = shape
    k = choice.shape[1]
    if not 1 <= k <= experts:
        raise RedistError(1, f"1 to {experts} experts can be chosen, not {k}")
    at = o.stream(device, stream)
    given = dlogits is not None
    if not given:
        dlogits = o.matrix(tokens, experts, dtype, device)
    places = (tokens, k)
    op = _pack_route(tokens, experts, k, _code(o, logits, "logits"), 1 if normalize else 0, logits.data_ptr(), *logits.stride(),
                     _table(o, weights, places, o.f32, device, "weights"), _table(o, choice, places, o.i32, device, "choice"), 0, 0)
    rc = o.route_backward(op, _table(o, dweights, places, o.f32, device, "dweights"), _pack_matrix(*_matrix(dlogits, shape, dtype, device, "dlogits")), at)
    if rc:
        raise RedistError(rc, "redist_route_backward")
    if given:
        o.written(dlogits)
    return dlogits


_ABSENT = (0, 0, 0)


def _move(o, token, row, position, residual=None, drow=None, weights=None, dweights=None):
    """The packed block of the four moves."""
    try:
        tokens, cols = token.shape
        rows, width = row.shape
        places, k = position.shape
    except ValueError:
        _not_matrices(tokens=token, rows=row, position=position)
        raise
    dtype, device, shape = token.dtype, token.device, (tokens, k)
    if width != cols or row.dtype is not dtype or row.device != device:
        _matrix(row, (rows, cols), dtype, device, "rows")                    # says what is wrong
    if places != tokens or position.dtype is not o.i32 or position.device != device or not position.is_contiguous():
        _table(o, position, shape, o.i32, device, "position")
    return _pack_move(tokens, rows, cols, _code(o, token, "tokens"), k, token.data_ptr(), *token.stride(), row.data_ptr(), *row.stride(),
                      *(_ABSENT if residual is None else _matrix(residual, (tokens, cols), dtype, device, "residual")),
                      *(_ABSENT if drow is None else _matrix(drow, (rows, cols), dtype, device, "drows")), position.data_ptr(),
                      0 if weights is None else _table(o, weights, shape, o.f32, device, "weights"),
                      0 if dweights is None else dweights.data_ptr())


def dispatch_forward(x, position, out=None, stream=None):
    """``redist_dispatch_forward``: every token of ``x`` (tokens, cols) in the rows that ``position`` (tokens, k) int32 names for
    it.  Returns ``out``, by default (tokens * k, cols); rows that nobody names are left as they were (in a new tensor: undefined).
    Row-major matrices in bfloat16, float16 or float32."""
    if stream is not None:
        with _allocating(stream):
            return _dispatch_forward(x, position, out, stream)
    return _dispatch_forward(x, position, out, None)


def _dispatch_forward(x, position, out, stream):
    o = _ops or _operators()
    at = o.stream(x.device, stream)
    given = out is not None
    if not given:
        if x.dim() != 2:
            _not_matrices(x=x)
        out = o.matrix(position.numel(), x.shape[1], x.dtype, x.device)
    rc = o.dispatch_forward(_move(o, x, out, position), at)
    if rc:
        raise RedistError(rc, "redist_dispatch_forward")
    if given:
        o.written(out)
    return out


def dispatch_backward(drows, position, dx=None, stream=None):
    """``redist_dispatch_backward``: ``dx`` (tokens, cols), a token's sum of its rows of ``drows`` (rows, cols)."""
    if stream is not None:
        with _allocating(stream):
            return _dispatch_backward(drows, position, dx, stream)
    return _dispatch_backward(drows, position, dx, None)


def _dispatch_backward(drows, position, dx, stream):
    o = _ops or _operators()
    at = o.stream(drows.device, stream)
    given = dx is not None
    if not given:
        if drows.dim() != 2:
            _not_matrices(drows=drows)
        dx = o.matrix(position.shape[0], drows.shape[1], drows.dtype, drows.device)
    rc = o.dispatch_backward(_move(o, dx, drows, position), at)
    if rc:
        raise RedistError(rc, "redist_dispatch_backward")
    if given:
        o.written(dx)
    return dx


def combine_forward(rows, position, weights=None, residual=None, out=None, stream=None):
    """``redist_combine_forward``: ``residual`` + the sum over a token's places of ``weights`` (tokens, k) float32 times the row of
    ``rows`` (rows, cols) that ``position`` names; without ``weights`` the plain sum.  ``out`` may be ``residual`` itself."""
    if stream is not None:
        with _allocating(stream):
            return _combine_forward(rows, position, weights, residual, out, stream)
    return _combine_forward(rows, position, weights, residual, out, None)


def _combine_forward(rows, position, weights, residual, out, stream):
    o = _ops or _operators()
    at = o.stream(rows.device, stream)
    given = out is not None
    if not given:
        if rows.dim() != 2:
            _not_matrices(rows=rows)
        out = o.matrix(position.shape[0], rows.shape[1], rows.dtype, rows.device)
    rc = o.combine_forward(_move(o, out, rows, position, residual, None, weights), at)
    if rc:
        raise RedistError(rc, "redist_combine_forward")
    if given:
        o.written(out)
    return out


def combine_backward(dy, rows, position, weights, drows=None, stream=None):
    """``redist_combine_backward``: ``(drows, dweights)`` -- ``weights`` times a token's ``dy`` (tokens, cols) in its rows, and the
    product of ``dy`` with each of them (float32, 0 in empty places).  Rows of ``drows`` that nobody names are left as they
    were (in a new tensor: undefined)."""
    if stream is not None:
        with _allocating(stream):
            return _combine_backward(dy, rows, position, weights, drows, stream)
    return _combine_backward(dy, rows, position, weights, drows, None)


def _combine_backward(dy, rows, position, weights, drows, stream):
    o = _ops or _operators()
    at = o.stream(dy.device, stream)
    given = drows is not None
    if not given:
        if rows.dim() != 2:
            _not_matrices(rows=rows)
        drows = o.matrix(rows.shape[0], rows.shape[1], rows.dtype, rows.device)
    if position.dim() != 2:
        _not_matrices(position=position)
    dweights = o.matrix(position.shape[0], position.shape[1], o.f32, dy.device)
    rc = o.combine_backward(_move(o, dy, rows, position, None, drows, weights, dweights), at)
    if rc:
        raise RedistError(rc, "redist_combine_backward")
    if given:
        o.written(drows)
    return drows, dweights


def _stack(t, shape, dtype, device, what: str):
    """``t`` as the fields of a redist_matrix and the distance from matrix to matrix, checked."""
    if t is None:
        return (0, 0, 0), 0
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        raise RedistError(1, f"{what} has to be {tuple(shape)} of {dtype} on {device}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
    apart, a, b = t.stride()
    return (t.data_ptr(), a, b), apart


def _not_stacks(**tensors) -> None:
    for name, t in tensors.items():
        if t.dim() != 3:
            raise RedistError(1, f"{name} has to be a stack of matrices, not of {t.dim()} dimensions")


def experts_forward(x, w, offsets, bias=None, activation: str = "none", out=None, pre=None, scratch=None, stream=None):
    """``redist_experts_forward``: the linear layer with a weight per range of rows, ``activation(x[r] @ w[e].T + bias[e])`` for
    rows ``offsets[e]`` to ``offsets[e + 1]``.

    ``x`` (rows, in) and ``w`` (experts, out, in), bfloat16 or float16; ``offsets`` (experts + 1,) int32 on the device, not
    decreasing; ``bias`` (experts, out) of any type; ``pre`` (rows, out), if given, receives ``x @ w.T + bias``.  Returns
    ``out`` (rows, out); rows of no expert are left as they were (in a new tensor: undefined)."""
    if stream is not None:
        with _allocating(stream):
            return _experts_forward(x, w, offsets, bias, activation, out, pre, scratch, stream)
    return _experts_forward(x, w, offsets, bias, activation, out, pre, scratch, None)


def _experts_forward(x, w, offsets, bias, activation, out, pre, scratch, stream):
    o = _ops or _operators()
    if x.dim() != 2 or w.dim() != 3:
        _not_matrices(x=x)
        _not_stacks(w=w)
    rows, k = x.shape
    experts, n = w.shape[0], w.shape[1]
    device, dtype, shape = x.device, x.dtype, (rows, n)
    at = o.stream(device, stream)
    given = out is not None
    if not given:
        out = o.matrix(rows, n, dtype, device)
    b, bt, bs = 0, 0, 0
    if bias is not None:
        if bias.shape != (experts, n) or bias.device != device or (n > 1 and bias.stride(1) != 1):
            raise RedistError(1, f"bias has to be {experts} x {n} with contiguous rows on {device}")
        b, bt, bs = bias.data_ptr(), _code(o, bias, "bias"), bias.stride(0)
    weight, apart = _stack(w, (experts, n, k), dtype, device, "w")
    op = _pack_experts(rows, k, n, experts, _code(o, x, "x"), bt, _activation(activation), x.data_ptr(), *x.stride(), *weight,
                       *_matrix(out, shape, dtype, device, "out"), *_matrix(pre, shape, dtype, device, "pre"), apart, bs, b,
                       _table(o, offsets, (experts + 1,), o.i32, device, "offsets"))
    rc = o.experts_forward(op, None, 0, at) if scratch is None else _ESCRATCH
    if rc == _ESCRATCH:                                      # operands off 16-byte boundaries: rare
        keep, sp, sn = o.scratch(o.experts_scratch_bytes(op, None), scratch, device)
        rc = o.experts_forward(op, sp, sn, at)
    if rc:
        raise RedistError(rc, "redist_experts_forward")
    if pre is not None or given:
        o.written([t for t in (pre, out if given else None) if t is not None])
    return out


def experts_backward(dy, x, w, offsets, pre=None, activation: str = "none", need=(True, True, True), dx=None, dw=None, dbias=None,
                     scratch=None, stream=None):
    """``redist_experts_backward``: ``(dx, dw, dbias)``, the gradients of :func:`experts_forward`; ``need`` says which of them are
    wanted.  dx (rows, in) and dw (experts, out, in) have the type of ``dy``, dbias (experts, out) is float32.  Experts
    without rows get zeros; rows of no expert are left as they were in dx (in a new tensor: undefined)."""
    if stream is not None:
        with _allocating(stream):
            return _experts_backward(dy, x, w, offsets, pre, activation, need, dx, dw, dbias, scratch, stream)
    return _experts_backward(dy, x, w, offsets, pre, activation, need, dx, dw, dbias, scratch, None)


def _experts_backward(dy, x, w, offsets, pre, activation, need, dx, dw, dbias, scratch, stream):
    o = _ops or _operators()
    if dy.dim() != 2 or x.dim() != 2 or w.dim() != 3:
        _not_matrices(dy=dy, x=x)
        _not_stacks(w=w)
    rows, n = dy.shape
    experts, k = w.shape[0], x.shape[1]
    device, dtype = dy.device, dy.dtype
    at = o.stream(device, stream)
    wide, tall, stack = (rows, n), (rows, k), (experts, n, k)
    given = [t for t, wanted in zip((dx, dw, dbias), need) if wanted and t is not None]
    if not need[0]:
        dx = None
    elif dx is None:
        dx = o.matrix(rows, k, dtype, device)
    if not need[1]:
        dw = None
    elif dw is None:
        dw = o.strided(stack, (n * k, k, 1), dtype=dtype, device=device)
    if not need[2]:
        dbias = None
    elif dbias is None:
        dbias = o.matrix(experts, n, o.f32, device)
    weight, apart = _stack(w, stack, dtype, device, "w")
    grad, grad_apart = _stack(dw, stack, dtype, device, "dw")
    op = _pack_experts(rows, k, n, experts, _code(o, dy, "dy"), 0, _activation(activation), *_matrix(x, tall, dtype, device, "x"), *weight, 0, 0, 0,
                       *_matrix(pre, wide, dtype, device, "pre"), apart, 0, 0, _table(o, offsets, (experts + 1,), o.i32, device, "offsets"))
    g = _pack_experts_grads(dy.data_ptr(), *dy.stride(), *_matrix(dx, tall, dtype, device, "dx"), *grad, grad_apart,
                            0 if dbias is None else _table(o, dbias, (experts, n), o.f32, device, "dbias"))
    keep, sp, sn = o.scratch(o.experts_scratch_bytes(op, g), scratch, device)
    rc = o.experts_backward(op, g, sp, sn, at)
    if rc:
        raise RedistError(rc, "redist_experts_backward")
    if given:
        o.written(given)
    return dx, dw, dbias


# ---- the bound on a step's gradients ---------------------------------------------------------------------


def _dense(t) -> bool:
    """Whether the elements of ``t`` lie side by side, in whatever order of the dimensions."""
    if t.is_contiguous():
        return True
    return t.permute(sorted(range(t.dim()), key=lambda d: (-t.stride(d), -t.shape[d]))).is_contiguous()


def clip_gradients(tensors, max_norm, eps: float = 1e-6, out=None, scratch=None, stream=None):
    """``redist_clip``: the norm over all elements of all ``tensors`` -- a 0-dimensional float32 tensor, returned -- and the
    tensors times ``min(1, max_norm / (norm + eps))``, in place or into the tensors of ``out`` (same shapes, strides and
    types).  ``max_norm`` None: the norm only.  bfloat16, float16 and float32 may be mixed; any shape whose elements lie
    side by side."""
    if stream is not None:
        with _allocating(stream):
            return _clip_gradients(tensors, max_norm, eps, out, scratch, stream)
    return _clip_gradients(tensors, max_norm, eps, out, scratch, None)


def _clip_gradients(tensors, max_norm, eps, out, scratch, stream):
    o = _ops or _operators()
    tensors = list(tensors)
    if max_norm is not None and not max_norm >= 0:
        raise RedistError(1, f"max_norm is not negative, or None, not {max_norm}")
    if out is not None:
        out = list(out)
        if len(out) != len(tensors):
            raise RedistError(1, f"{len(tensors)} tensors, but {len(out)} to write")
    device = tensors[0].device if tensors else o.torch.device("cuda", o.current_device() if o.current_device else 0)
    at = o.stream(device, stream)
    # (a list may be long: what can be asked of all tensors at once is)
    T, n, codes = o.torch.Tensor, len(tensors), o.codes
    if any(map(device.index.__ne__, map(T.get_device, tensors))) or not (all(map(T.is_contiguous, tensors)) or all(map(_dense, tensors))):
        raise RedistError(1, "gradients have to be on one device, the elements of each side by side")
    types = [codes.get(t.dtype) for t in tensors]
    if None in types:
        _code(o, tensors[types.index(None)], "a gradient")
    table = array.array("q", bytes(32 * n))                  # entries of four words: data, out, elements, type and reserved
    table[0::4] = array.array("q", list(map(T.data_ptr, tensors)))
    table[2::4] = array.array("q", list(map(T.numel, tensors)))
    table[3::4] = array.array("q", types)
    if out is not None:
        for i, (t, v) in enumerate(zip(tensors, out)):
            if v.shape != t.shape or v.dtype is not t.dtype or v.device != device or v.stride() != t.stride():
                raise RedistError(1, f"out has to be like the gradients; number {i} is not")
        table[1::4] = array.array("q", list(map(T.data_ptr, out)))
    norm = o.strided((), (), dtype=o.f32, device=device)
    op = _pack_clip(table.buffer_info()[0], n, -1.0 if max_norm is None else max_norm, eps, norm.data_ptr())
    keep, sp, sn = o.scratch(o.clip_scratch_bytes(op), scratch, device)
    rc = o.clip(op, sp, sn, at)
    if rc:
        raise RedistError(rc, "redist_clip")
    if max_norm is not None and tensors:
        o.written(tensors if out is None else out)
    return norm


def redist_product_timeouts() -> int:
    """Thread blocks of the matrix products whose bounded wait ran out on the current device (0 in a healthy run)."""
    return int(load().redist_product_timeouts())
