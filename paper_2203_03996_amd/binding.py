"""ctypes binding of libdeltacnn.so: same names as the C ABI, argument marshalling only.

PyTorch is used for device memory (`torch.empty(..., device="cuda")`) and for the HIP
stream; every step of the path runs inside the library's kernels.  There is no CPU
fallback: importing works without a GPU (so the symbol table can be checked), but creating
a context without the built library or without an MI355X raises.
"""
from __future__ import annotations

import ctypes as C
import os
import threading
from dataclasses import dataclass

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libdeltacnn.so")

F32, F16, BF16, I8 = range(4)          # (BF16 and I8: row operators only)
DELTAGEN, CONV, DWCONV, ACT, MAXPOOL, UPSAMPLE, ACCUM, CONCAT, UPSAMPLE_BILINEAR, GAVGPOOL = range(10)
ACT_NONE, ACT_RELU, ACT_RELU6 = 0, 1, 2
ACT_CODES = {"none": ACT_NONE, None: ACT_NONE, "relu": ACT_RELU, "relu6": ACT_RELU6}
TORCH_DTYPE = {F32: torch.float32, F16: torch.float16}
ROW_DTYPE_CODE = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
NORM_CODES = {"none": 0, None: 0, "rms": 1, "layer": 2}
ROT_CODES = {"halves": 0, "pairs": 1}
DTYPE_CODE = {"f32": F32, "f16": F16}
STATUS_NAMES = ["OK", "EINVAL", "ESHAPE", "EDTYPE", "ESTATE", "ENOMEM", "EHIP", "EUNSUPPORTED"]

EXPORTS = [
    "dcnn_workspace_bytes", "dcnn_ctx_create", "dcnn_ctx_destroy", "dcnn_ctx_sync", "dcnn_status_str",
    "dcnn_last_error", "dcnn_mask_compact", "dcnn_mask_compact_static", "dcnn_layer_query", "dcnn_layer_create", "dcnn_layer_destroy",
    "dcnn_layer_init", "dcnn_layer_step", "dcnn_layer_output", "dcnn_layer_reset", "dcnn_layer_state",
    "dcnn_layer_stats", "dcnn_layer_set_eps", "dcnn_layer_set_timing", "dcnn_layer_set_counting", "dcnn_layer_timing", "dcnn_net_create", "dcnn_net_destroy", "dcnn_net_add", "dcnn_net_finalize",
    "dcnn_net_bind", "dcnn_net_init", "dcnn_net_step", "dcnn_net_reset", "dcnn_net_output",
    "dcnn_net_num_layers", "dcnn_net_layer", "dcnn_net_stats",
    "dcnn_rows_norm", "dcnn_rows_weights_bytes", "dcnn_rows_pack", "dcnn_rows_scratch_bytes", "dcnn_rows_matmul",
    "dcnn_rows_linear", "dcnn_rows_heads", "dcnn_cache_append", "dcnn_cache_read", "dcnn_cache_scratch_bytes", "dcnn_cache_attend",
]


class DeltaStruct(C.Structure):
    _fields_ = [("data", C.c_void_p), ("mask", C.c_void_p), ("idx", C.c_void_p), ("count", C.c_void_p),
                ("n", C.c_int32), ("h", C.c_int32), ("w", C.c_int32), ("c", C.c_int32), ("dtype", C.c_int32)]


class LayerDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("dtype", C.c_int32), ("n", C.c_int32), ("h", C.c_int32), ("w", C.c_int32),
                ("c", C.c_int32), ("kh", C.c_int32), ("kw", C.c_int32), ("stride", C.c_int32), ("pad", C.c_int32),
                ("cout", C.c_int32), ("act", C.c_int32), ("eps", C.c_float), ("n_in", C.c_int32),
                ("dilate_r", C.c_int32), ("factor", C.c_int32), ("want_idx", C.c_int32),
                ("proj_c", C.c_int32), ("proj_h", C.c_int32), ("proj_w", C.c_int32), ("proj_stride", C.c_int32),
                ("fuse_accum", C.c_int32), ("no_xT", C.c_int32), ("xT_residue", C.c_int32)]


class LayerSizes(C.Structure):
    _fields_ = [("state_bytes", C.c_size_t), ("on", C.c_int32), ("oh", C.c_int32), ("ow", C.c_int32),
                ("oc", C.c_int32)]


class Stats(C.Structure):
    _fields_ = [("pixels_in", C.c_int64), ("pixels_in2", C.c_int64), ("pixels_work", C.c_int64),
                ("pixels_out", C.c_int64), ("pixels_total", C.c_int64), ("pixels_in_total", C.c_int64),
                ("pixels_in2_total", C.c_int64),
                ("kind", C.c_int32), ("act", C.c_int32), ("n_in", C.c_int32), ("c_in", C.c_int32),
                ("c_out", C.c_int32), ("k", C.c_int32), ("stride", C.c_int32), ("proj_c", C.c_int32), ("fuse_accum", C.c_int32),
                ("reserved", C.c_int32), ("xT_bytes_read", C.c_int64), ("xT_bytes_written", C.c_int64)]

    def as_dict(self) -> dict:
        return {name: getattr(self, name) for name, _ in self._fields_ if name != "reserved"}


# (nested members -- dcnn_row_list, dcnn_row_norm -- are spelled out: an attribute of a nested structure costs an object)
_ROW_LIST = [("rows", C.c_int64), ("map_rows", C.c_int64), ("idx", C.c_void_p), ("count", C.c_void_p)]


def _row_norm(name):
    return [(name + "_kind", C.c_int32), (name + "_eps", C.c_float), (name + "_w", C.c_void_p), (name + "_b", C.c_void_p)]


class RowsNormArgs(C.Structure):
    _fields_ = _ROW_LIST + [
        ("dtype", C.c_int32), ("c", C.c_int32), ("x", C.c_void_p), ("h", C.c_void_p), ("gate", C.c_void_p),
        ("y", C.c_void_p), ("z", C.c_void_p), ("q", C.c_void_p), ("q_scale", C.c_void_p), ("ldx", C.c_int64),
        ("ldh", C.c_int64), ("ldg", C.c_int64), ("ldy", C.c_int64), ("ldz", C.c_int64), ("ldq", C.c_int64),
        ("gate_rows", C.c_int64), ("scale", C.c_float), ("_pad", C.c_int32)] + _row_norm("post") + _row_norm("pre")


class RowsMatmulArgs(C.Structure):
    _fields_ = _ROW_LIST + [
        ("dtype", C.c_int32), ("act", C.c_int32), ("k", C.c_int64), ("n", C.c_int64), ("packed", C.c_void_p),
        ("bias", C.c_void_p), ("y", C.c_void_p), ("ldy", C.c_int64), ("q", C.c_void_p), ("q_scale", C.c_void_p),
        ("ldq", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64)] + _row_norm("pre") + [
        ("scratch", C.c_void_p), ("scratch_bytes", C.c_size_t)]


_TOKENS = _ROW_LIST + [("period", C.c_int64), ("stream", C.c_void_p), ("pos", C.c_void_p)]
_ROTATION = [("table", C.c_void_p), ("positions", C.c_int64), ("rot", C.c_int32), ("style", C.c_int32)]
_CACHE = [("dtype", C.c_int32), ("heads", C.c_int32), ("dim", C.c_int32), ("page", C.c_int32), ("streams", C.c_int64), ("length", C.c_int64),
          ("num_pages", C.c_int64), ("codes", C.c_void_p), ("scales", C.c_void_p), ("pages", C.c_void_p)]


class RowsHeadsArgs(C.Structure):
    _fields_ = _TOKENS + [
        ("dtype", C.c_int32), ("dim", C.c_int32), ("q_heads", C.c_int32), ("k_heads", C.c_int32), ("q", C.c_void_p), ("k", C.c_void_p),
        ("q_out", C.c_void_p), ("k_out", C.c_void_p), ("ldq", C.c_int64), ("ldk", C.c_int64), ("ldq_out", C.c_int64),
        ("ldk_out", C.c_int64)] + _row_norm("q_norm") + _row_norm("k_norm") + _ROTATION


class CacheAppendArgs(C.Structure):
    _fields_ = _CACHE + _TOKENS + [("k", C.c_void_p), ("v", C.c_void_p), ("ldk", C.c_int64), ("ldv", C.c_int64)] + _row_norm("k_norm") + _ROTATION


class CacheReadArgs(C.Structure):
    _fields_ = _CACHE + _TOKENS + [("k_out", C.c_void_p), ("v_out", C.c_void_p), ("ldk", C.c_int64), ("ldv", C.c_int64)]


class CacheAttendArgs(C.Structure):
    _fields_ = _CACHE + _TOKENS + [
        ("q", C.c_void_p), ("y", C.c_void_p), ("ldq", C.c_int64), ("ldy", C.c_int64), ("q_heads", C.c_int32), ("scale", C.c_float),
        ("causal", C.c_int32), ("_pad", C.c_int32), ("window", C.c_int64), ("lens", C.c_void_p), ("scratch", C.c_void_p), ("scratch_bytes", C.c_size_t)]


class DcnnError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"libdeltacnn: {STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else status}: {text}")
        self.status = status


_lib = None


def load_library() -> C.CDLL:
    """Load the built shared library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                                "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
    P = C.POINTER
    lib.dcnn_workspace_bytes.restype = sz
    lib.dcnn_workspace_bytes.argtypes = [C.c_int64]
    lib.dcnn_ctx_create.argtypes = [vp, vp, sz, P(vp)]
    lib.dcnn_ctx_destroy.argtypes = [vp]
    lib.dcnn_ctx_destroy.restype = None
    lib.dcnn_ctx_sync.argtypes = [vp]
    lib.dcnn_status_str.restype = C.c_char_p
    lib.dcnn_status_str.argtypes = [i32]
    lib.dcnn_last_error.restype = C.c_char_p
    lib.dcnn_last_error.argtypes = [vp]
    lib.dcnn_mask_compact.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp]
    lib.dcnn_mask_compact_static.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, vp, vp]
    lib.dcnn_layer_query.argtypes = [P(LayerDesc), P(LayerSizes)]
    lib.dcnn_layer_create.argtypes = [vp, P(LayerDesc), vp, vp, vp, sz, P(vp)]
    lib.dcnn_layer_destroy.argtypes = [vp]
    lib.dcnn_layer_destroy.restype = None
    lib.dcnn_layer_init.argtypes = [vp, P(vp), i32, vp]
    lib.dcnn_layer_step.argtypes = [vp, P(P(DeltaStruct)), i32]
    lib.dcnn_layer_output.argtypes = [vp, P(DeltaStruct)]
    lib.dcnn_layer_reset.argtypes = [vp]
    lib.dcnn_layer_state.argtypes = [vp, i32, P(vp), P(sz)]
    lib.dcnn_layer_stats.argtypes = [vp, P(Stats)]
    lib.dcnn_layer_set_eps.argtypes = [vp, C.c_float]
    lib.dcnn_layer_set_timing.argtypes = [vp, i32]
    lib.dcnn_layer_set_counting.argtypes = [vp, i32]
    lib.dcnn_layer_timing.argtypes = [vp, P(C.c_float), P(i32)]
    lib.dcnn_net_create.argtypes = [vp, i32, i32, i32, i32, i32, P(vp)]
    lib.dcnn_net_destroy.argtypes = [vp]
    lib.dcnn_net_destroy.restype = None
    lib.dcnn_net_add.argtypes = [vp, P(LayerDesc), P(i32), i32, vp, vp, P(i32)]
    lib.dcnn_net_finalize.argtypes = [vp, i32, P(sz)]
    lib.dcnn_net_bind.argtypes = [vp, vp, sz]
    lib.dcnn_net_init.argtypes = [vp, vp, vp]
    lib.dcnn_net_step.argtypes = [vp, vp, vp]
    lib.dcnn_net_reset.argtypes = [vp]
    lib.dcnn_net_output.argtypes = [vp, P(DeltaStruct)]
    lib.dcnn_net_num_layers.argtypes = [vp]
    lib.dcnn_net_num_layers.restype = i32
    lib.dcnn_net_layer.argtypes = [vp, i32, P(vp), P(i32)]
    lib.dcnn_net_stats.argtypes = [vp, P(Stats)]
    lib.dcnn_rows_norm.argtypes = [vp, P(RowsNormArgs)]
    lib.dcnn_rows_weights_bytes.argtypes = [C.c_int64, C.c_int64]
    lib.dcnn_rows_weights_bytes.restype = sz
    lib.dcnn_rows_pack.argtypes = [vp, i32, C.c_int64, C.c_int64, vp, C.c_int64, vp, vp, sz]
    lib.dcnn_rows_scratch_bytes.argtypes = [C.c_int64, C.c_int64, C.c_int64, i32]
    lib.dcnn_rows_scratch_bytes.restype = sz
    lib.dcnn_rows_matmul.argtypes = [vp, P(RowsMatmulArgs)]
    lib.dcnn_rows_linear.argtypes = [vp, P(RowsMatmulArgs)]
    lib.dcnn_rows_heads.argtypes = [vp, P(RowsHeadsArgs)]
    lib.dcnn_cache_append.argtypes = [vp, P(CacheAppendArgs)]
    lib.dcnn_cache_read.argtypes = [vp, P(CacheReadArgs)]
    lib.dcnn_cache_scratch_bytes.argtypes = [i32, C.c_int64, i32, i32, i32, C.c_int64, C.c_int64]
    lib.dcnn_cache_scratch_bytes.restype = sz
    lib.dcnn_cache_attend.argtypes = [vp, P(CacheAttendArgs)]
    _lib = lib
    return lib


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


@dataclass
class Delta:
    """Device tensors of one sparse update (see dcnn_delta in deltacnn.h)."""
    data: torch.Tensor            # [n,h,w,c]
    mask: torch.Tensor | None     # uint8 [n,h,w]
    idx: torch.Tensor | None      # int32 [n*h*w]
    count: torch.Tensor | None    # int32 [1]

    def struct(self) -> DeltaStruct:
        n, h, w, c = self.data.shape
        code = F16 if self.data.dtype == torch.float16 else F32
        return DeltaStruct(_ptr(self.data), _ptr(self.mask), _ptr(self.idx), _ptr(self.count), n, h, w, c, code)


class Context:
    """dcnn_ctx on torch's current stream, with a torch-allocated workspace.

    All calls run on that stream, whichever torch is on later: tensors made on another one are the caller's to wait for.  Calls
    on one context follow each other (one thread at a time), with its GPU as torch's current one."""

    def __init__(self, max_pixels: int, device="cuda"):
        """max_pixels = 0 creates the context without a workspace (enough for mask_compact_static)."""
        self.lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("libdeltacnn needs an MI355X (gfx950); no GPU is visible and there is no CPU path")
        self.device = torch.device(device)
        nbytes = self.lib.dcnn_workspace_bytes(int(max_pixels)) if max_pixels > 0 else 0
        self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=self.device) if nbytes else None
        self.stream = torch.cuda.current_stream(self.device)
        self.index, self._raw_stream = self.stream.device_index, self.stream.cuda_stream
        self._gpu = torch.device("cuda", self.index)
        h = C.c_void_p()
        st = self.lib.dcnn_ctx_create(C.c_void_p(self.stream.cuda_stream), C.c_void_p(_ptr(self.workspace)),
                                      nbytes, C.byref(h))
        if st != 0:
            raise DcnnError(st, self.lib.dcnn_status_str(st).decode())
        self.handle = h
        self._bases = []          # tensors whose memory library-returned pointers may point into

    def check(self, st: int):
        if st != 0:
            raise DcnnError(st, self.lib.dcnn_last_error(self.handle).decode())

    def sync(self):
        self.check(self.lib.dcnn_ctx_sync(self.handle))

    def register(self, *tensors):
        for t in tensors:
            if t is not None:
                self._bases.append(t)

    def view(self, ptr: int, nbytes: int, dtype, shape):
        """Torch view of library-returned device memory that lies inside a registered tensor."""
        for b in self._bases:
            lo = b.data_ptr()
            if lo <= ptr and ptr + nbytes <= lo + b.numel() * b.element_size():
                flat = b.reshape(-1).view(torch.uint8)
                return flat[ptr - lo:ptr - lo + nbytes].view(dtype).reshape(shape)
        raise ValueError("pointer does not belong to a registered tensor")

    def delta_view(self, s: DeltaStruct) -> Delta:
        dt = TORCH_DTYPE[s.dtype]
        px = s.n * s.h * s.w
        es = 2 if s.dtype == F16 else 4
        return Delta(self.view(s.data, px * s.c * es, dt, (s.n, s.h, s.w, s.c)),
                     self.view(s.mask, px, torch.uint8, (s.n, s.h, s.w)) if s.mask else None,
                     self.view(s.idx, px * 4, torch.int32, (px,)) if s.idx else None,
                     self.view(s.count, 4, torch.int32, (1,)) if s.count else None)

    def mask_compact(self, mask_in, k=1, stride=1, pad=0, mask_b=None):
        n, h, w = mask_in.shape
        oh, ow = (h + 2 * pad - k) // stride + 1, (w + 2 * pad - k) // stride + 1
        mask_out = torch.empty((n, oh, ow), dtype=torch.uint8, device=self.device)
        idx = torch.empty(n * oh * ow, dtype=torch.int32, device=self.device)
        count = torch.empty(1, dtype=torch.int32, device=self.device)
        self.check(self.lib.dcnn_mask_compact(self.handle, _ptr(mask_in), n, h, w, k, stride, pad, _ptr(mask_b),
                                              _ptr(mask_out), _ptr(idx), _ptr(count)))
        return mask_out, idx, count

    def mask_compact_static(self, mask_in, mask_out, idx, count, k=1, stride=1, pad=0, mask_b=None):
        """dcnn_mask_compact_static: the caller passes every output buffer (mask_out may be None); the call
        itself allocates nothing."""
        n, h, w = mask_in.shape
        self.check(self.lib.dcnn_mask_compact_static(self.handle, _ptr(mask_in), n, h, w, k, stride, pad, _ptr(mask_b),
                                                     _ptr(mask_out), _ptr(idx), _ptr(count)))

    def empty(self, shape, dtype):
        """An uninitialised device tensor that belongs to the context's GPU and stream, whichever torch is on."""
        # (torch.cuda.current_stream builds an object, 3 us; the calls that allocate their outputs take 8 in all)
        if torch._C._cuda_getCurrentRawStream(self.index) == self._raw_stream:
            return torch.empty(shape, dtype=dtype, device=self._gpu)
        with torch.cuda.stream(self.stream):
            return torch.empty(shape, dtype=dtype, device=self._gpu)

    def capturing(self) -> bool:
        """Whether a graph is being captured on the context's stream, whichever stream torch is on."""
        if torch._C._cuda_getCurrentRawStream(self.index) == self._raw_stream and torch.cuda.current_device() == self.index:
            return torch.cuda.is_current_stream_capturing()
        with torch.cuda.stream(self.stream):
            return torch.cuda.is_current_stream_capturing()

    def rows_norm(self, x=None, h=None, *, post=None, gate=None, gate_rows=0, scale=1.0, pre=None, idx=None, count=None,
                  y=None, z=None, q=None, q_scale=None):
        """dcnn_rows_norm: y = x + scale * gate * post(h) and z = pre(y), z also in 8 bits (q with q_scale).

        x and y are maps (last dimension c), the rest is [rows, c].  y, z, q: a tensor to write, True for a new one, or
        None where it is not wanted (q_scale: a tensor [rows], or None for a new one).  post, pre: RowNorm or None.
        Rows that a list does not name are left as they are (in a new y: uninitialised).  Without a count all rows of x,
        or all that idx names, are wanted: a matrix with fewer is refused.  With a count the smallest of idx, h, z and q
        is the room of the call, and what the count names beyond it is left as it is too.
        Returns (y, z, q, q_scale)."""
        t = h if x is None else x
        if t is None:
            raise ValueError("rows_norm: neither x nor h")
        c, dt, dev = t.shape[-1], t.dtype, self.index
        a = RowsNormArgs()
        a.dtype, a.c, a.scale = _row_dtype(dt), c, scale
        rows = map_rows = None
        if idx is not None:
            a.idx, rows = _int32(idx, "idx", dev), idx.numel()
        if count is not None:
            a.count = _int32(count, "count", dev)
        if x is not None:
            a.x, a.ldx, map_rows = _as_rows(x, "x", c, dt, dev)
            if rows is None:
                rows = map_rows
        if h is not None:
            a.h, a.ldh, n = _as_rows(h, "h", c, dt, dev)
            rows = n if rows is None else _room(rows, n, "h", count)
        if y is not None:
            if y is True:
                y = self.empty((rows, c) if x is None else x.shape, dt)
            a.y, a.ldy, n = _as_rows(y, "y", c, dt, dev)
            if map_rows is not None and n != map_rows:
                raise ValueError(f"rows_norm: x has {map_rows} rows, y {n}")
            map_rows = n
        elif x is None:
            map_rows = rows if idx is None else 0x7fffffff
        if gate is not None:
            a.gate, a.ldg, n = _as_rows(gate, "gate", c, dt, dev) if gate.dim() > 1 else (_vector(gate, "gate", c, dt, dev), c, 1)
            a.gate_rows = gate_rows
            if n < (-(-map_rows // gate_rows) if gate_rows > 0 else 1):
                raise ValueError(f"rows_norm: {n} rows of gate for {map_rows} map rows, {gate_rows} to each")
        if z is not None:
            if z is True:
                z = self.empty((rows, c), dt)
                a.z, a.ldz = z.data_ptr(), c
            else:
                a.z, a.ldz, n = _as_rows(z, "z", c, dt, dev)
                rows = _room(rows, n, "z", count)
        if q is not None:
            if q is True:
                q = self.empty((rows, -(-c // 16) * 16), torch.int8)[:, :c]
            if q_scale is None:
                q_scale = self.empty(rows, torch.float32)
            a.q, a.q_scale, a.ldq = _check_q(q, q_scale, c, dev)
            rows = _room(rows, q.shape[0], "q", count)
        if post is not None:
            a.post_kind, a.post_eps, a.post_w, a.post_b = post.pointers(c, dt, dev)
        if pre is not None:
            a.pre_kind, a.pre_eps, a.pre_w, a.pre_b = pre.pointers(c, dt, dev)
        a.rows, a.map_rows = rows, map_rows
        st = self.lib.dcnn_rows_norm(self.handle, a)
        if st:
            self.check(st)
        return y, z, q, q_scale

    def rows_heads(self, q, k=None, *, dim, q_norm=None, k_norm=None, rotation=None, positions=None, idx=None, count=None, q_out=None, k_out=None):
        """dcnn_rows_heads: queries q [rows, heads * dim] and keys k, each head normed by itself and rotated by the row's position.

        A row's token is map row i = idx[r] (r without a list); its position is positions[i], or i counted round and round the
        rotation's table (maps of as many pixels).  q_norm, k_norm: RowNorm over `dim` values, or None; rotation: Rotation or
        None.  q_out, k_out: a matrix to write (q and k themselves: in place), or None for a new one.  Without a count every row
        that idx names is wanted; with one the smallest matrix is the room of the call.  Returns (q_out, k_out), or q_out alone
        without keys."""
        a, dt, dev = RowsHeadsArgs(), q.dtype, self.index
        a.dtype, a.dim = _row_dtype(dt), dim
        a.q, a.ldq, rows, c = _matrix(q, "q", dim, 0, dt, dev)
        a.q_heads = c // dim
        period = 1
        if rotation is not None:
            period = rotation.positions
            a.table, a.positions, a.rot, a.style = rotation.pointers(dev)
        rows = _set_tokens(a, rows, None, positions, period, idx, count, dev)
        if k is not None:
            a.k, a.ldk, n, ck = _matrix(k, "k", dim, 0, dt, dev)
            a.k_heads = ck // dim
            if n < rows:
                rows = _room(rows, n, "k", count)
        if q_out is not None:
            a.q_out, a.ldq_out, n, _ = _matrix(q_out, "q_out", dim, c, dt, dev)
            rows = _room(rows, n, "q_out", count)
        if k_out is not None and k is not None:
            a.k_out, a.ldk_out, n, _ = _matrix(k_out, "k_out", dim, ck, dt, dev)
            rows = _room(rows, n, "k_out", count)
        if q_out is None:
            q_out = self.empty((rows, c), dt)
            a.q_out, a.ldq_out = q_out.data_ptr(), c
        if k_out is None and k is not None:
            k_out = self.empty((rows, ck), dt)
            a.k_out, a.ldk_out = k_out.data_ptr(), ck
        if q_norm is not None:
            a.q_norm_kind, a.q_norm_eps, a.q_norm_w, a.q_norm_b = q_norm.pointers(dim, dt, dev)
        if k_norm is not None:
            a.k_norm_kind, a.k_norm_eps, a.k_norm_w, a.k_norm_b = k_norm.pointers(dim, dt, dev)
        a.rows = rows
        st = self.lib.dcnn_rows_heads(self.handle, a)
        if st:
            self.check(st)
        return q_out if k is None else (q_out, k_out)

    def rows_quantize(self, x, *, pre=None, idx=None, count=None):
        """Rows of x (normed with `pre`, or as they are) in 8 bits: (q [rows, c], q_scale [rows])."""
        return self.rows_norm(x, pre=pre, idx=idx, count=count, q=True)[2:]

    def __del__(self):
        try:
            if getattr(self, "handle", None):
                self.lib.dcnn_ctx_destroy(self.handle)
                self.handle = None
        except Exception:
            pass


def make_desc(kind, dtype, n, h, w, c, k=1, stride=1, pad=0, cout=0, act=ACT_NONE, eps=0.0, n_in=1, dilate_r=0,
              factor=1, want_idx=1, proj=None, fuse_accum=0, no_xT=0, xT_residue=0) -> LayerDesc:
    """proj = (channels, height, width, stride) of the input of a fused 1x1 projection shortcut, or None."""
    pc, ph, pw, ps = proj if proj is not None else (0, 0, 0, 0)
    return LayerDesc(kind, dtype, n, h, w, c, k, k, stride, pad, cout, act, float(eps), n_in, dilate_r, factor,
                     want_idx, pc, ph, pw, ps, fuse_accum, int(no_xT), int(xT_residue))


class Layer:
    """dcnn_layer with torch-allocated state memory."""

    def __init__(self, ctx: Context, desc: LayerDesc, weights: torch.Tensor | None = None,
                 bias: torch.Tensor | None = None):
        self.ctx, self.desc = ctx, desc
        lib = ctx.lib
        sizes = LayerSizes()
        st = lib.dcnn_layer_query(C.byref(desc), C.byref(sizes))
        if st != 0:
            raise DcnnError(st, lib.dcnn_status_str(st).decode())
        self.out_shape = (sizes.on, sizes.oh, sizes.ow, sizes.oc)
        self.state = torch.zeros(sizes.state_bytes, dtype=torch.uint8, device=ctx.device)
        ctx.register(self.state)
        h = C.c_void_p()
        ctx.check(lib.dcnn_layer_create(ctx.handle, C.byref(desc), _ptr(weights), _ptr(bias), _ptr(self.state),
                                        sizes.state_bytes, C.byref(h)))
        self.handle = h
        self._keep = (weights, bias)

    def init(self, dense_in, dense_out=None):
        d = self.desc
        if not dense_in or tuple(dense_in[0].shape) != (d.n, d.h, d.w, d.c):
            raise ValueError(f"dense input 0 must have shape {(d.n, d.h, d.w, d.c)}")
        for t in dense_in:
            if t.dtype != TORCH_DTYPE[d.dtype] or not t.is_contiguous() or not t.is_cuda:
                raise ValueError("dense inputs must be contiguous device tensors of the layer's type")
        arr = (C.c_void_p * len(dense_in))(*[t.data_ptr() for t in dense_in])
        if dense_out is None and self.desc.kind != ACCUM:
            dense_out = torch.empty(self.out_shape, dtype=TORCH_DTYPE[self.desc.dtype], device=self.ctx.device)
        self.ctx.check(self.ctx.lib.dcnn_layer_init(self.handle, arr, len(dense_in), _ptr(dense_out)))
        return dense_out

    def step(self, inputs):
        structs = [d.struct() for d in inputs]
        for d in inputs:
            self.ctx.register(d.data, d.mask, d.idx, d.count)
        arr = (C.POINTER(DeltaStruct) * len(structs))(*[C.pointer(s) for s in structs])
        self.ctx.check(self.ctx.lib.dcnn_layer_step(self.handle, arr, len(structs)))
        return self.output()

    def output(self) -> Delta:
        s = DeltaStruct()
        self.ctx.check(self.ctx.lib.dcnn_layer_output(self.handle, C.byref(s)))
        return self.ctx.delta_view(s)

    def reset(self):
        self.ctx.check(self.ctx.lib.dcnn_layer_reset(self.handle))

    def set_eps(self, eps: float):
        self.ctx.check(self.ctx.lib.dcnn_layer_set_eps(self.handle, float(eps)))

    def state_tensor(self, which: int) -> torch.Tensor:
        p, n = C.c_void_p(), C.c_size_t()
        self.ctx.check(self.ctx.lib.dcnn_layer_state(self.handle, which, C.byref(p), C.byref(n)))
        dt = TORCH_DTYPE[self.desc.dtype]
        d = self.desc
        shape = (d.n, d.h, d.w, d.c) if d.kind in (DELTAGEN, MAXPOOL) else self.out_shape
        return self.ctx.view(p.value, n.value, dt, shape)

    def stats(self) -> dict:
        s = Stats()
        self.ctx.check(self.ctx.lib.dcnn_layer_stats(self.handle, C.byref(s)))
        return s.as_dict()

    def set_timing(self, max_steps: int):
        """Record HIP events around the layer's main kernel for the next `max_steps` steps (0: off)."""
        self.ctx.check(self.ctx.lib.dcnn_layer_set_timing(self.handle, max_steps))

    def timing(self):
        """(summed kernel milliseconds, launches) since the last call."""
        ms, n = C.c_float(), C.c_int32()
        self.ctx.check(self.ctx.lib.dcnn_layer_timing(self.handle, C.byref(ms), C.byref(n)))
        return ms.value, n.value

    def __del__(self):
        try:
            if getattr(self, "handle", None):
                self.ctx.lib.dcnn_layer_destroy(self.handle)
                self.handle = None
        except Exception:
            pass


_ROWS_MAX = 0x7fffffff                     # of a map or a compact matrix
_SCRATCH_ROWS = 64                         # linear products of more rows take scratch of their own


def _row_dtype(dt) -> int:
    code = ROW_DTYPE_CODE.get(dt)
    if code is None:
        raise ValueError(f"row operators take float32, float16 and bfloat16, got {dt}")
    return code


def _as_rows(t, name, c, dt, dev):
    """(address, leading dimension, rows) of a tensor as a matrix of c columns; the ABI takes bare pointers, so shapes are checked here."""
    if t.dim() != 2:
        t = t.view(-1, t.shape[-1])
    n, cols = t.shape
    if cols != c or t.dtype is not dt or t.get_device() != dev:
        raise ValueError(f"{name} must hold rows of {c} {dt} on GPU {dev}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    if n <= 1 or t.is_contiguous():
        if c > 1 and t.stride(1) != 1:
            raise ValueError(f"{name}: the elements of a row must lie side by side (strides {t.stride()})")
        return t.data_ptr(), c, n
    ld, one = t.stride()
    if ld < c or (one != 1 and c > 1):
        raise ValueError(f"{name}: rows of {c} elements side by side, apart from each other (strides {t.stride()})")
    return t.data_ptr(), ld, n


def _room(rows, n, name, count):
    """Rows of a call with a compact matrix of n rows: it may have fewer than the call where their number is on the GPU, and nowhere else."""
    if n >= rows:
        return rows
    if count is None:
        raise ValueError(f"{name} has {n} rows, {rows} are wanted")
    return n


def _vector(t, name, c, dt, dev):
    if t.numel() != c or t.dtype is not dt or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [{c}] {dt} on GPU {dev}, got {tuple(t.shape)} {t.dtype}")
    return t.data_ptr()


def _check_q(q, q_scale, c, dev):
    """(address, address of the scales, leading dimension) of 8-bit rows."""
    if q.dim() != 2 or q.shape[1] != c or q.dtype != torch.int8 or q.get_device() != dev or (c > 1 and q.stride(1) != 1):
        raise ValueError(f"q must be an int8 device matrix of {c} columns, got {tuple(q.shape)} {q.dtype} strides {q.stride()}")
    n, padded = q.shape[0], -(-c // 16) * 16
    if q_scale.dtype != torch.float32 or q_scale.numel() < n or not q_scale.is_contiguous() or q_scale.get_device() != dev:
        raise ValueError(f"q_scale must hold {n} float32 numbers on the device")
    ld = q.stride(0) if n > 1 else padded
    if c != padded and n and q.storage_offset() + (n - 1) * ld + padded > q.untyped_storage().nbytes():
        raise ValueError("the last row of q does not fill its multiple of 16 bytes")
    return q.data_ptr(), q_scale.data_ptr(), ld


def _int32(t, name, dev):
    if t.dtype != torch.int32 or not t.is_contiguous() or t.get_device() != dev or (name == "count" and t.numel() != 1):
        raise ValueError(f"{name} must be a contiguous int32 device tensor")
    return t.data_ptr()


class RowNorm:
    """A norm over a row's channels: kind "rms" or "layer", weight and bias [c] (None: ones, zeros), which it keeps.

    Each call reads the parameters where they lie then: a module's may move or change their type between calls."""

    def __init__(self, kind: str, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, eps: float = 1e-5):
        self.kind, self.weight, self.bias, self.eps = NORM_CODES[kind], weight, bias, float(eps)
        for t in (weight, bias):
            if t is not None and (t.dim() != 1 or not t.is_contiguous()):
                raise ValueError(f"a norm's parameters must be contiguous vectors, got {tuple(t.shape)} strides {t.stride()}")

    def pointers(self, c: int, dt, dev):
        """(kind, eps, address of the weight, address of the bias) for rows of c channels."""
        w, b = self.weight, self.bias
        return (self.kind, self.eps, None if w is None else _vector(w, "a norm's weight", c, dt, dev),
                None if b is None else _vector(b, "a norm's bias", c, dt, dev))


class RowWeights:
    """Weights [k, n] of a product, in 8 bits with a scale per output channel, laid out once for the matrix cores (dcnn_rows_pack).

    weights: floating point (quantised here), or int8 with `scale` [n].  bias: [n] of the outputs' type, or None; each call reads
    it where it lies then.

    The object holds scratch that its calls share, as large as the 8-bit rows of its largest linear call (a list's: as many rows
    as the list has room for).  Calls follow each other on the context's stream, and threads take turns.  Graphs hold the scratch
    too: two that were captured from one object must not run at the same time, and the object has to outlive them."""

    def __init__(self, ctx: Context, weights: torch.Tensor, scale: torch.Tensor | None = None, bias: torch.Tensor | None = None, act="none"):
        self.ctx, lib = ctx, ctx.lib
        if weights.dim() != 2 or weights.stride(1) != 1 or weights.get_device() != ctx.index:
            raise ValueError(f"weights must be a matrix [k, n] on GPU {ctx.index}, the elements of a row side by side")
        k, n = weights.shape
        code = I8 if weights.dtype == torch.int8 else _row_dtype(weights.dtype)
        if (scale is not None) != (code == I8) or (scale is not None and (scale.shape != (n,) or scale.dtype != torch.float32 or
                                                                          not scale.is_contiguous() or scale.get_device() != ctx.index)):
            raise ValueError(f"8-bit weights come with a float32 scale [{n}] on GPU {ctx.index}, others without one")
        self.k, self.n, self.bias = k, n, bias
        nbytes = lib.dcnn_rows_weights_bytes(k, n)
        if nbytes == 0:
            raise ValueError(f"weights [{k}, {n}] are out of range")
        self.packed = ctx.empty(nbytes, torch.uint8)
        ctx.check(lib.dcnn_rows_pack(ctx.handle, code, k, n, weights.data_ptr(), weights.stride(0) if k > 1 else n, _ptr(scale),
                                     self.packed.data_ptr(), nbytes))
        for t in (weights, scale):                                # (their memory is theirs until the stream has read them)
            if t is not None:
                t.record_stream(ctx.stream)
        if bias is not None and (bias.shape != (n,) or not bias.is_contiguous() or bias.get_device() != ctx.index):
            raise ValueError(f"bias must be a contiguous tensor [{n}] on GPU {ctx.index}")
        self.act = ACT_CODES[act]
        # scratch for all products of 8-bit rows (partial sums: 8 MB at most) and the linear ones of few rows
        nbytes = max(lib.dcnn_rows_scratch_bytes(_ROWS_MAX, k, n, 0), lib.dcnn_rows_scratch_bytes(_SCRATCH_ROWS, k, n, 1))
        with torch.cuda.stream(ctx.stream):
            self._scratch = torch.zeros(nbytes, dtype=torch.uint8, device=ctx._gpu)
        self._scratch_at = self._scratch.data_ptr(), nbytes
        self._grown, self._grown_rows, self._captured = None, 0, set()         # _captured: what graphs hold the address of
        self._one_call = threading.Lock()

    def _call(self, call, linear, a, rows, dt, count, out):
        ctx = self.ctx
        a.dtype, a.k, a.n, a.act, a.packed = _row_dtype(dt), self.k, self.n, self.act, self.packed.data_ptr()
        if self.bias is not None:                                 # (where it lies now, as the outputs' type is this call's)
            a.bias = _vector(self.bias, "bias", self.n, dt, ctx.index)
        if count is not None:
            a.count = _int32(count, "count", ctx.index)
        if out is None:
            out = ctx.empty((rows, self.n), dt)
            a.y, a.ldy = out.data_ptr(), self.n
        else:
            a.y, a.ldy, n = _as_rows(out, "out", self.n, dt, ctx.index)
            rows = _room(rows, n, "out", count)
        a.rows = rows
        with self._one_call:                                      # (a call's kernels follow each other: both use the scratch)
            a.scratch, a.scratch_bytes = self._scratch_at if not linear or rows <= _SCRATCH_ROWS else self._linear_scratch(rows)
            st = call(ctx.handle, a)
            if st:
                ctx.check(st)
        return out

    def _linear_scratch(self, rows):
        """(address, bytes) of scratch that holds so many 8-bit rows; a larger one takes the place of a smaller one."""
        capturing = self.ctx.capturing()
        scratch = self._grown
        if scratch is None or rows > self._grown_rows:
            need = self.ctx.lib.dcnn_rows_scratch_bytes(rows, self.k, self.n, 1)
            with torch.cuda.stream(self.ctx.stream):
                scratch = torch.zeros(need, dtype=torch.uint8, device=self.ctx._gpu)
            if not capturing:                                     # (else it is the graph's: the kernel that clears it runs when the graph does)
                self._grown, self._grown_rows = scratch, rows
        elif capturing:
            self._captured.add(scratch)
        return scratch.data_ptr(), scratch.numel()

    def matmul(self, q, q_scale, *, dtype=torch.float16, count=None, out=None):
        """dcnn_rows_matmul: the product of 8-bit rows [rows, k] with a scale each, [rows, n] of `dtype`.

        out: a matrix to write, of `rows` rows at least; with a count it may have fewer (what the count names beyond them is not computed)."""
        a = RowsMatmulArgs()
        a.q, a.q_scale, a.ldq = _check_q(q, q_scale, self.k, self.ctx.index)
        return self._call(self.ctx.lib.dcnn_rows_matmul, 0, a, q.shape[0], dtype, count, out)

    def linear(self, x, *, pre=None, idx=None, count=None, out=None):
        """dcnn_rows_linear: rows of the map x (those that idx names), normed with `pre`, quantised and multiplied; [rows, n].  out: as in matmul."""
        a, dt, dev = RowsMatmulArgs(), x.dtype, self.ctx.index
        a.x, a.ldx, rows = _as_rows(x, "x", self.k, dt, dev)
        a.map_rows = rows
        if idx is not None:
            a.idx, rows = _int32(idx, "idx", dev), idx.numel()
        if pre is not None:
            a.pre_kind, a.pre_eps, a.pre_w, a.pre_b = pre.pointers(self.k, dt, dev)
        return self._call(self.ctx.lib.dcnn_rows_linear, 1, a, rows, dt, count, out)


def _matrix(t, name, dim, c, dt, dev):
    """(address, leading dimension, rows, columns) of a matrix of heads of `dim` values, of c columns if c is not 0."""
    if t.dim() != 2 or t.dtype is not dt or t.get_device() != dev:
        raise ValueError(f"{name} must be a matrix of {dt} on GPU {dev}, got {tuple(t.shape)} {t.dtype} on {t.device}")
    n, cols = t.shape
    ld, one = t.stride()
    if cols != c if c else cols == 0 or cols % dim:
        raise ValueError(f"{name} must have {c or f'heads * {dim}'} columns, got {tuple(t.shape)}")
    if one != 1 or (ld < cols and n > 1):
        raise ValueError(f"{name}: rows of {cols} elements side by side, apart from each other (strides {t.stride()})")
    return t.data_ptr(), ld if n > 1 else cols, n, cols


def _set_tokens(a, n, streams, positions, period, idx, count, dev):
    """Fills in which tokens the rows of an n-row matrix are; returns the rows of the call so far."""
    a.period, rows, known = period, n, None
    if positions is not None:
        a.pos, known = _int32(positions, "positions", dev), positions.numel()
    if streams is not None:
        a.stream, m = _int32(streams, "streams", dev), streams.numel()
        known = m if known is None or m < known else known
    if idx is not None:
        a.idx, rows = _int32(idx, "idx", dev), idx.numel()
        a.map_rows = _ROWS_MAX if known is None else known
    elif known is None:
        a.map_rows = n
    else:
        if known < n:
            raise ValueError(f"{known} streams or positions for a matrix of {n} rows")
        a.map_rows = known
    if count is not None:
        a.count = _int32(count, "count", dev)
    return rows if n >= rows else _room(rows, n, "a matrix of rows", count)


class Rotation:
    """Rotation of heads by position: `table` [positions, rot / 2, 2] float32, the cosine and sine of each pair's angle.

    style "halves": pair j is the values j and j + rot / 2 of a head; "pairs": 2 j and 2 j + 1.  Values from rot on are left alone."""

    def __init__(self, table: torch.Tensor, style: str = "halves"):
        if table.dim() != 3 or table.shape[2] != 2 or table.dtype != torch.float32 or not table.is_contiguous() or table.shape[1] % 8 or not table.numel():
            raise ValueError(f"a rotation's table must be contiguous float32 [positions, a multiple of 8, 2], got {tuple(table.shape)} {table.dtype}")
        self.table, self.style, self.positions, self.rot = table, ROT_CODES[style], table.shape[0], 2 * table.shape[1]

    @classmethod
    def of_angles(cls, angles: torch.Tensor, style: str = "halves"):
        """From angles [positions, rot / 2] (float64: those of far positions need it)."""
        a = angles.double()
        return cls(torch.stack([a.cos(), a.sin()], 2).float().contiguous(), style)

    @classmethod
    def of_positions(cls, positions: int, rot: int, base: float = 10000.0, style: str = "halves", device="cuda"):
        """Pair j turns by position * base ^ (-2 j / rot)."""
        p = torch.arange(positions, dtype=torch.float64, device=device)[:, None]
        return cls.of_angles(p * base ** (-torch.arange(rot // 2, dtype=torch.float64, device=device) * 2 / rot), style)

    @classmethod
    def of_pixels(cls, h: int, w: int, rot: int, base: float = 100.0, style: str = "halves", device="cuda"):
        """Pixels of an h x w map: the first half of the pairs turns by the row, the second by the column (rot a multiple of 16)."""
        f = base ** (-torch.arange(rot // 4, dtype=torch.float64, device=device) * 4 / rot)
        y, x = (torch.arange(n, dtype=torch.float64, device=device)[:, None] * f for n in (h, w))
        return cls.of_angles(torch.cat([y[:, None].expand(h, w, -1), x[None].expand(h, w, -1)], 2).reshape(h * w, -1), style)

    def pointers(self, dev):
        if self.table.get_device() != dev:
            raise ValueError(f"the rotation's table is on {self.table.device}, the call on GPU {dev}")
        return self.table.data_ptr(), self.positions, self.rot, self.style


class TokenCache:
    """Keys and values of the tokens of `streams` streams, up to `length` each, in 4 bits (dcnn_cache), and attention over them.

    heads, dim: of keys and values; dtype: of queries, keys, values and outputs.  page: tokens of a page.  pages: int32
    [streams, ceil(length / page)], the number of each page, read at every call (to hand pages out anew, write into it), or
    None where every stream has its own, one behind the other.  codes, scales: the memory (see dcnn_cache), or None for
    new, zeroed memory of `num_pages` pages (as many as all streams need where it is not given).

    Calls name tokens as rows: map row i = idx[r] (r without a list) is a token of streams[i] at positions[i].  Without both
    the maps are pixels, `length` to a stream: stream i / length, position i % length; with positions alone row i is the
    token of stream i.  Matrices are compact; without a count every row that idx names is wanted.

    The object holds scratch that its attend calls share, as large as the largest of them needs or up to half as large again.
    Calls follow each other on the context's stream, and threads take turns.  Graphs hold the scratch too (one that has grown
    since stays for them): two that were captured from one object must not run at the same time, and the object has to
    outlive them."""

    def __init__(self, ctx: Context, streams: int, length: int, heads: int, dim: int, *, dtype=torch.float16, page: int = 64, pages=None,
                 num_pages: int | None = None, codes: torch.Tensor | None = None, scales: torch.Tensor | None = None):
        self.ctx, self.streams, self.length, self.heads, self.dim, self.page = ctx, streams, length, heads, dim, page
        self.dtype, self._code = dtype, _row_dtype(dtype)
        if min(streams, length, heads, dim) < 1 or page < 16 or page > 4096 or page & (page - 1) or dim % 32:
            raise ValueError(f"a cache of {streams} streams of {length} tokens, {heads} heads of {dim}, pages of {page}")
        per_stream = -(-length // page)
        if (codes is None) != (scales is None):
            raise ValueError("codes and scales come together")
        if codes is None:
            num_pages = streams * per_stream if num_pages is None else num_pages
            with torch.cuda.stream(ctx.stream):
                codes, scales = (torch.zeros((num_pages, 2, heads, page, n), dtype=torch.uint8, device=ctx._gpu) for n in (dim // 2, dim // 32))
        elif num_pages is not None and num_pages != codes.shape[0]:
            raise ValueError(f"{num_pages} pages, codes of {codes.shape[0]}")
        self.num_pages = codes.shape[0]
        for name, t, n in (("codes", codes, dim // 2), ("scales", scales, dim // 32)):
            if t.shape != (self.num_pages, 2, heads, page, n) or t.dtype != torch.uint8 or not t.is_contiguous() or t.get_device() != ctx.index:
                raise ValueError(f"{name} must be contiguous uint8 [pages, 2, {heads}, {page}, {n}] on GPU {ctx.index}, got {tuple(t.shape)} {t.dtype} on {t.device}")
        if pages is not None and (pages.shape != (streams, per_stream) or pages.dtype != torch.int32 or not pages.is_contiguous() or pages.get_device() != ctx.index):
            raise ValueError(f"pages must be contiguous int32 [{streams}, {per_stream}] on GPU {ctx.index}, got {tuple(pages.shape)} {pages.dtype}")
        if pages is None and self.num_pages < streams * per_stream:
            raise ValueError(f"{self.num_pages} pages for {streams} streams of {per_stream}")
        self.codes, self.scales, self.pages = codes, scales, pages
        # (_captured: scratch that graphs hold the address of, kept when a larger one takes its place; _in_graph: whether what is there now is among it)
        self._scratch, self._scratch_at, self._in_graph, self._captured, self._needs, self._one_call = None, (0, 0), False, [], {}, threading.Lock()

    def _args(self, a, n, streams, positions, idx, count):
        """Fills in the cache and the tokens of a call with an n-row matrix; returns its rows."""
        a.dtype, a.heads, a.dim, a.page = self._code, self.heads, self.dim, self.page
        a.streams, a.length, a.num_pages = self.streams, self.length, self.num_pages
        a.codes, a.scales = self.codes.data_ptr(), self.scales.data_ptr()
        if self.pages is not None:
            a.pages = self.pages.data_ptr()
        if positions is None:
            if streams is not None:
                raise ValueError("streams come with positions")
            return _set_tokens(a, n, None, None, self.length, idx, count, self.ctx.index)
        return _set_tokens(a, n, streams, positions, 1, idx, count, self.ctx.index)

    def append(self, k, v, *, norm: RowNorm | None = None, rotation: Rotation | None = None, streams=None, positions=None, idx=None, count=None):
        """dcnn_cache_append: keys k [rows, heads * dim] (normed and rotated on the way) and values v into their tokens' places,
        which must be distinct."""
        a, ctx, c = CacheAppendArgs(), self.ctx, self.heads * self.dim
        dev = ctx.index
        a.k, a.ldk, n, _ = _matrix(k, "k", self.dim, c, self.dtype, dev)
        rows = self._args(a, n, streams, positions, idx, count)
        a.v, a.ldv, n, _ = _matrix(v, "v", self.dim, c, self.dtype, dev)
        a.rows = rows if n >= rows else _room(rows, n, "v", count)
        if norm is not None:
            a.k_norm_kind, a.k_norm_eps, a.k_norm_w, a.k_norm_b = norm.pointers(self.dim, self.dtype, dev)
        if rotation is not None:
            a.table, a.positions, a.rot, a.style = rotation.pointers(dev)
        st = ctx.lib.dcnn_cache_append(ctx.handle, a)
        if st:
            ctx.check(st)

    def read(self, *, streams=None, positions=None, idx=None, count=None, rows: int | None = None):
        """dcnn_cache_read: (keys, values) [rows, heads * dim] that the cache holds for tokens, zeros for those it has no place for.

        The tokens are those that idx names, else as many as positions has, else the first `rows` of all (None: all)."""
        if idx is not None:
            n = idx.numel()
        elif positions is not None:
            n = positions.numel()
        else:
            n = self.streams * self.length if rows is None else rows
        a, ctx, c = CacheReadArgs(), self.ctx, self.heads * self.dim
        a.rows = self._args(a, n, streams, positions, idx, count)
        k, v = ctx.empty((2, n, c), self.dtype).unbind()
        a.k_out, a.v_out, a.ldk, a.ldv = k.data_ptr(), v.data_ptr(), c, c
        st = ctx.lib.dcnn_cache_read(ctx.handle, a)
        if st:
            ctx.check(st)
        return k, v

    def attend(self, q, *, lens=None, causal=False, window: int = 0, scale: float | None = None, streams=None, positions=None, idx=None, count=None, out=None):
        """dcnn_cache_attend: attention of queries q [rows, q_heads * dim] over the tokens of their streams, [rows, q_heads * dim].

        q_heads is a multiple of the cache's heads; consecutive query heads share one.  lens: int32 [streams], the tokens that
        count (None: `length`).  causal: none behind the row's position; window: only those nearer to it than so many (0: all).
        scale: of the products, 1 / sqrt(dim) where it is None.  out: a matrix to write."""
        a, ctx = CacheAttendArgs(), self.ctx
        dev = ctx.index
        a.q, a.ldq, n, c = _matrix(q, "q", self.dim, 0, self.dtype, dev)
        rows = self._args(a, n, streams, positions, idx, count)
        if out is None:
            out = ctx.empty((rows, c), self.dtype)
            a.y, a.ldy = out.data_ptr(), c
        else:
            a.y, a.ldy, n, _ = _matrix(out, "out", self.dim, c, self.dtype, dev)
            rows = _room(rows, n, "out", count)
        if lens is not None:
            a.lens = _int32(lens, "lens", dev)
            if lens.numel() < self.streams:
                raise ValueError(f"lens of {lens.numel()} streams, the cache has {self.streams}")
        q_heads = c // self.dim
        a.rows, a.q_heads, a.window = rows, q_heads, window
        if causal:
            a.causal = 1
        a.scale = self.dim ** -0.5 if scale is None else scale
        need = self._needs.get((rows, q_heads))
        if need is None:
            need = ctx.lib.dcnn_cache_scratch_bytes(self._code, rows, q_heads, self.heads, self.dim, self.streams, self.length)
            if len(self._needs) < 4096:
                self._needs[rows, q_heads] = need
        with self._one_call:                                      # (a call's kernels follow each other: both use the scratch)
            scratch = None
            if need > self._scratch_at[1]:
                scratch = self._larger_scratch(need)              # (a graph's own is held until the call is recorded)
                a.scratch, a.scratch_bytes = scratch.data_ptr(), scratch.numel()
            else:
                a.scratch, a.scratch_bytes = self._scratch_at
                if not self._in_graph and ctx.capturing():        # (once: a graph holds it from now on)
                    self._in_graph = True
                    self._captured.append(self._scratch)
            st = ctx.lib.dcnn_cache_attend(ctx.handle, a)
            if st:
                ctx.check(st)
        return out

    def _larger_scratch(self, need):
        """New scratch: it takes the place of the one before it, half as large again at least, so that sizes that rise by a little are made anew now and
        then only.  While a graph is being captured it is the graph's alone, out of the graph's memory."""
        if self.ctx.capturing():
            return self.ctx.empty(need, torch.uint8)
        scratch = self.ctx.empty(max(need, self._scratch_at[1] * 3 // 2), torch.uint8)
        self._scratch, self._scratch_at, self._in_graph = scratch, (scratch.data_ptr(), scratch.numel()), False
        return scratch


_KIND = {"deltagen": DELTAGEN, "act": ACT, "add": ACT, "maxpool": MAXPOOL, "upsample": UPSAMPLE, "accum": ACCUM}


class Net:
    """dcnn_net built from a topology table (dict with "nodes", "dtype", "h", "w", "c"; see
    the header for node kinds) and a dict {node index: (weights, bias)} of numpy arrays."""

    def __init__(self, ctx: Context, spec: dict, weights: dict, n_streams: int, flags: int = 1):
        self.ctx, self.spec = ctx, spec
        lib = ctx.lib
        self.dtype = DTYPE_CODE[spec["dtype"]]
        tdt = TORCH_DTYPE[self.dtype]
        self.n = int(n_streams)
        h = C.c_void_p()
        ctx.check(lib.dcnn_net_create(ctx.handle, self.dtype, self.n, spec["h"], spec["w"], spec["c"], C.byref(h)))
        self.handle = h
        self._weights = {}
        for i, nd in enumerate(spec["nodes"]):
            kind = nd["kind"]
            wdev = bdev = None
            if kind == "conv":
                wgt, bias = weights[i]
                # one direct round-to-nearest-even to the storage type (numpy's conversion; going through
                # float32 first, as torch's float64 -> float16 does, rounds twice)
                ndt = np.float16 if self.dtype == F16 else np.float32
                wdev = torch.from_numpy(np.ascontiguousarray(np.asarray(wgt).astype(ndt))).to(ctx.device)
                bdev = torch.from_numpy(np.ascontiguousarray(np.asarray(bias).astype(ndt))).to(ctx.device)
                self._weights[i] = (wdev, bdev)
                desc = make_desc(DWCONV if nd["depthwise"] else CONV, self.dtype, 0, 0, 0, 0, k=nd["k"],
                                 stride=nd["stride"], pad=nd["pad"], cout=nd["cout"])
            elif kind == "deltagen":
                desc = make_desc(DELTAGEN, self.dtype, 0, 0, 0, 0, eps=nd["eps"], dilate_r=nd.get("dilate_r", 0))
            elif kind == "act":
                desc = make_desc(ACT, self.dtype, 0, 0, 0, 0, act=ACT_CODES[nd["f"]], eps=nd["eps"], n_in=1,
                                 no_xT=1 if nd.get("no_xT") else 0, xT_residue=1 if nd.get("xT_residue") else 0)
            elif kind == "add":
                desc = make_desc(ACT, self.dtype, 0, 0, 0, 0, act=ACT_NONE, n_in=2)
            elif kind == "concat":
                desc = make_desc(CONCAT, self.dtype, 0, 0, 0, 0, n_in=2)
            elif kind == "maxpool":
                desc = make_desc(MAXPOOL, self.dtype, 0, 0, 0, 0, k=nd["k"], stride=nd["stride"], pad=nd["pad"])
            elif kind == "upsample":
                desc = make_desc(UPSAMPLE, self.dtype, 0, 0, 0, 0, factor=nd["factor"])
            elif kind == "upsample_bilinear":
                desc = make_desc(UPSAMPLE_BILINEAR, self.dtype, 0, 0, 0, 0, factor=nd["factor"])
            elif kind == "gavgpool":
                desc = make_desc(GAVGPOOL, self.dtype, 0, 0, 0, 0)
            elif kind == "accum":
                desc = make_desc(ACCUM, self.dtype, 0, 0, 0, 0)
            else:
                raise ValueError(kind)
            ins = (C.c_int32 * max(1, len(nd["in"])))(*nd["in"])
            nid = C.c_int32()
            ctx.check(lib.dcnn_net_add(self.handle, C.byref(desc), ins, len(nd["in"]), _ptr(wdev), _ptr(bdev),
                                       C.byref(nid)))
            assert nid.value == i
        nbytes = C.c_size_t()
        ctx.check(lib.dcnn_net_finalize(self.handle, flags, C.byref(nbytes)))
        self.arena = torch.zeros(nbytes.value, dtype=torch.uint8, device=ctx.device)
        ctx.register(self.arena)
        ctx.check(lib.dcnn_net_bind(self.handle, _ptr(self.arena), nbytes.value))
        ctx.sync()                      # weights have been packed into the arena
        self.num_layers = lib.dcnn_net_num_layers(self.handle)

    def _check_frame(self, frame: torch.Tensor, out: torch.Tensor | None):
        # the ABI takes bare pointers: a tensor of the wrong size would be read or written out of bounds
        want = (self.n, self.spec["h"], self.spec["w"], self.spec["c"])
        if tuple(frame.shape) != want or frame.dtype != TORCH_DTYPE[self.dtype] or not frame.is_contiguous() or not frame.is_cuda:
            raise ValueError(f"frame must be a contiguous device tensor {want} of {TORCH_DTYPE[self.dtype]}, got "
                             f"{tuple(frame.shape)} {frame.dtype}")
        if out is not None and (out.dtype != TORCH_DTYPE[self.dtype] or not out.is_contiguous() or not out.is_cuda or
                                out.shape[0] != self.n):
            raise ValueError("out must be a contiguous device tensor [n, h, w, c] of the network's type")

    def init(self, frame: torch.Tensor, out: torch.Tensor | None = None):
        self._check_frame(frame, out)
        self.ctx.check(self.ctx.lib.dcnn_net_init(self.handle, _ptr(frame), _ptr(out)))

    def step(self, frame: torch.Tensor, out: torch.Tensor | None = None):
        self._check_frame(frame, out)
        self.ctx.check(self.ctx.lib.dcnn_net_step(self.handle, _ptr(frame), _ptr(out)))

    def reset(self):
        self.ctx.check(self.ctx.lib.dcnn_net_reset(self.handle))

    def output(self) -> Delta:
        s = DeltaStruct()
        self.ctx.check(self.ctx.lib.dcnn_net_output(self.handle, C.byref(s)))
        return self.ctx.delta_view(s)

    def layer_output(self, i: int):
        """(node id, Delta view, raw handle) of layer i of the fused plan."""
        lh, nid = C.c_void_p(), C.c_int32()
        self.ctx.check(self.ctx.lib.dcnn_net_layer(self.handle, i, C.byref(lh), C.byref(nid)))
        s = DeltaStruct()
        self.ctx.check(self.ctx.lib.dcnn_layer_output(lh, C.byref(s)))
        return nid.value, self.ctx.delta_view(s), lh

    def layer_state(self, i: int, which: int):
        lh, nid = C.c_void_p(), C.c_int32()
        self.ctx.check(self.ctx.lib.dcnn_net_layer(self.handle, i, C.byref(lh), C.byref(nid)))
        p, n = C.c_void_p(), C.c_size_t()
        st = self.ctx.lib.dcnn_layer_state(lh, which, C.byref(p), C.byref(n))
        if st != 0:
            return None
        es = 2 if self.dtype == F16 else 4
        return self.ctx.view(p.value, n.value, TORCH_DTYPE[self.dtype], (n.value // es,))

    def stats(self):
        arr = (Stats * self.num_layers)()
        self.ctx.check(self.ctx.lib.dcnn_net_stats(self.handle, arr))
        return [s.as_dict() for s in arr]

    def layer_node(self, i: int) -> int:
        """Node of the topology table whose output planned layer i produces."""
        lh, nid = C.c_void_p(), C.c_int32()
        self.ctx.check(self.ctx.lib.dcnn_net_layer(self.handle, i, C.byref(lh), C.byref(nid)))
        return nid.value

    def set_eps(self, i: int, eps: float):
        """New truncation threshold for planned layer i (input layer or a layer with an activation)."""
        lh, nid = C.c_void_p(), C.c_int32()
        self.ctx.check(self.ctx.lib.dcnn_net_layer(self.handle, i, C.byref(lh), C.byref(nid)))
        self.ctx.check(self.ctx.lib.dcnn_layer_set_eps(lh, float(eps)))

    def set_timing(self, i: int, max_steps: int):
        lh, nid = C.c_void_p(), C.c_int32()
        self.ctx.check(self.ctx.lib.dcnn_net_layer(self.handle, i, C.byref(lh), C.byref(nid)))
        self.ctx.check(self.ctx.lib.dcnn_layer_set_timing(lh, max_steps))

    def set_counting(self, on: bool):
        """Statistics mode for every layer: steps also count the x^T rows read / written (see dcnn_stats)."""
        for i in range(self.num_layers):
            lh, nid = C.c_void_p(), C.c_int32()
            self.ctx.check(self.ctx.lib.dcnn_net_layer(self.handle, i, C.byref(lh), C.byref(nid)))
            self.ctx.check(self.ctx.lib.dcnn_layer_set_counting(lh, 1 if on else 0))

    def timing(self, i: int):
        """(summed kernel milliseconds, launches) of layer i since the last call."""
        lh, nid = C.c_void_p(), C.c_int32()
        self.ctx.check(self.ctx.lib.dcnn_net_layer(self.handle, i, C.byref(lh), C.byref(nid)))
        ms, n = C.c_float(), C.c_int32()
        self.ctx.check(self.ctx.lib.dcnn_layer_timing(lh, C.byref(ms), C.byref(n)))
        return ms.value, n.value

    def __del__(self):
        try:
            if getattr(self, "handle", None):
                self.ctx.lib.dcnn_net_destroy(self.handle)
                self.handle = None
        except Exception:
            pass
