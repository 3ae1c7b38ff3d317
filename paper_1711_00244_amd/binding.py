"""ctypes binding over libcompressed_layer.so: argument marshalling only.

Every step of the path (decode, prefix sums, codebook lookup, multiply) runs in
the library's HIP kernels.  Tensors are torch CUDA tensors used as raw device
memory; the stream is torch's current stream.  There is no fallback: if the
library is missing or was not built, importing a symbol from it raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os

import numpy as np

from . import build as _build

CL_OK, CL_EINVAL, CL_ENOMEM, CL_ECORRUPT, CL_EUNSUPPORTED, CL_EHIP = 0, -1, -2, -3, -4, -5
PATH_AUTO, PATH_SPARSE, PATH_MFMA_F32, PATH_MFMA_BF16, PATH_SPARSE_WIDE = 0, 1, 2, 3, 4
CHUNK_BITS, RECORD_BITS, RECORDS_PER_CHUNK, MAX_RECORD_ENTRIES, MAX_CODE_LEN = 4096, 64, 64, 15, 12
STATIC_SCRATCH_BYTES = 16 << 20        # CL_STATIC_SCRATCH_BYTES
MX4 = 3                                # CL_MX4, after the element types of _element_type
ACTIVATIONS = {"none": 0, "relu": 1, "gated": 2}
SCORES = {"softmax": 0, "sigmoid": 1}
GROUP_SCORES = {"max": 0, "top2": 1}
MX_FORMS = ("few", "rows", "tile 64", "tile 128", "tile 256 x 128", "tile 256")       # CL_MX_FORM_*

EXPORTS = [
    "cl_last_error", "cl_compress_layer", "cl_layer_upload", "cl_layer_free", "cl_layer_stats",
    "cl_layer_host_view", "cl_layer_serialize", "cl_layer_deserialize", "cl_decode_layer",
    "cl_fc_workspace_bytes", "cl_fc_resolved_path", "cl_compressed_fc_forward", "cl_compressed_fc_forward_static", "cl_fc_stack_workspace_bytes",
    "cl_compressed_fc_stack_forward", "cl_layer_group_create", "cl_layer_group_free", "cl_fc_group_workspace_bytes",
    "cl_compressed_fc_group_forward", "cl_conv_workspace_bytes", "cl_conv_workspace_bytes_min", "cl_conv_workspace_bytes_unsplit",
    "cl_compressed_conv_forward", "cl_plan_batches", "cl_maxpool_forward", "cl_lrn_forward",
    "cl_set_kernel_timing", "cl_last_kernel_ms",
    "cl_mx_quantize", "cl_mx_dequantize", "cl_mx_fc_workspace_bytes", "cl_mx_fc_forward", "cl_route_experts", "cl_expert_lists_bytes",
    "cl_expert_lists", "cl_mx_experts_workspace_bytes", "cl_mx_experts_forward", "cl_mx_fc_resolved_form", "cl_mx_experts_resolved_form",
]


class LayerDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("M", "K", "weight_bits", "index_bits", "block_h", "block_w", "chunk_bits", "max_code_len")]


class Stats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("nnz", "padding", "entries", "n_blocks", "n_chunks", "val_bits", "idx_bits",
                                         "val_bits_unlimited", "idx_bits_unlimited", "n_records", "payload_bytes", "table_bytes",
                                         "model_bytes", "lut_bytes")] + [("val_max_len", C.c_int32), ("idx_max_len", C.c_int32)]


class ChunkMeta(C.Structure):
    _fields_ = [("sym_off", C.c_uint32), ("rec_off", C.c_uint32), ("blk", C.c_uint32), ("pos0", C.c_uint32)]


class HostView(C.Structure):
    _fields_ = [("desc", LayerDesc), ("codebook", C.POINTER(C.c_float)), ("val_len", C.POINTER(C.c_uint8)),
                ("val_code", C.POINTER(C.c_uint32)), ("idx_len", C.POINTER(C.c_uint8)), ("idx_code", C.POINTER(C.c_uint32)),
                ("block_ptr", C.POINTER(C.c_uint32)), ("panel_chunk", C.POINTER(C.c_uint32)),
                ("chunk_meta", C.POINTER(ChunkMeta)), ("records", C.POINTER(C.c_uint64)),
                ("n_blocks", C.c_int64), ("n_chunks", C.c_int64), ("n_records", C.c_int64), ("n_entries", C.c_int64),
                ("n_panels", C.c_int32), ("chunk_nz", C.POINTER(C.c_uint32)), ("max_block_nnz", C.c_int64),
                ("max_group_blocks", C.c_int32), ("chunk_half", C.POINTER(C.c_uint32)), ("group_ptr", C.POINTER(C.c_uint32))]


class ConvDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("C", "H", "W", "R", "S", "stride", "pad", "groups", "out_channels")]


class MxMatrix(C.Structure):
    _fields_ = [("d_codes", C.c_void_p), ("d_scales", C.c_void_p), ("rows", C.c_int32), ("K", C.c_int32)]


class MxInput(C.Structure):
    _fields_ = [("d_X", C.c_void_p), ("d_scales", C.c_void_p), ("type", C.c_int32), ("stride", C.c_int64)]


class RouteDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("experts", "k", "score", "groups", "groups_kept", "group_score", "renormalize")] + [("scale", C.c_float)]


class MxExpertsCall(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("k", C.c_int32), ("d_experts", C.c_void_p), ("d_weights", C.c_void_p), ("d_bias", C.c_void_p),
                ("d_lists", C.c_void_p), ("act", C.c_int32), ("x_per_pair", C.c_int32)]


class CLError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"[{code}] {msg}")
        self.code = code


_lib = None


def library_path() -> str:
    return _build.LIB


def lib():
    """Load the built library; build it only if no built library is there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB):
        _build.build_library()
    # PyTorch brings a HIP runtime of its own, and device memory comes from PyTorch: its
    # runtime has to be the one in the process before this library resolves its HIP
    # symbols (loaded the other way round, PyTorch afterwards finds no GPU)
    try:
        import torch  # noqa: F401
    except ImportError:
        pass
    L = C.CDLL(_build.LIB)
    p, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    L.cl_last_error.restype = C.c_char_p
    L.cl_compress_layer.argtypes = [C.POINTER(LayerDesc), p, p, C.POINTER(p)]
    L.cl_layer_upload.argtypes = [p]
    L.cl_layer_free.argtypes = [p]
    L.cl_layer_stats.argtypes = [p, C.POINTER(Stats)]
    L.cl_layer_host_view.argtypes = [p, C.POINTER(HostView)]
    L.cl_layer_serialize.argtypes = [p, p, C.POINTER(sz)]
    L.cl_layer_deserialize.argtypes = [p, sz, C.POINTER(p)]
    L.cl_decode_layer.argtypes = [p, p, p, p, p, p]
    L.cl_fc_workspace_bytes.argtypes = [p, i32, i32, C.POINTER(sz)]
    L.cl_fc_resolved_path.argtypes = [p, i32, i32, C.POINTER(i32)]
    L.cl_compressed_fc_forward_static.argtypes = [p, p, p, p, i32, i32, i32, p]
    L.cl_compressed_fc_forward.argtypes = [p, p, p, p, i32, i32, i32, p, sz, p]
    L.cl_fc_stack_workspace_bytes.argtypes = [p, i32, i32, i32, C.POINTER(sz)]
    L.cl_compressed_fc_stack_forward.argtypes = [p, i32, p, p, p, i32, i32, i32, i32, p, sz, p]
    L.cl_layer_group_create.argtypes = [p, i32, C.POINTER(p)]
    L.cl_fc_group_workspace_bytes.argtypes = [p, i32, C.POINTER(sz)]
    L.cl_compressed_fc_group_forward.argtypes = [p, p, sz, p, sz, p, i32, i32, p, sz, p]
    L.cl_conv_workspace_bytes.argtypes = [p, C.POINTER(ConvDesc), i32, i32, C.POINTER(sz)]
    L.cl_conv_workspace_bytes_min.argtypes = [p, C.POINTER(ConvDesc), i32, i32, C.POINTER(sz)]
    L.cl_conv_workspace_bytes_unsplit.argtypes = [p, C.POINTER(ConvDesc), i32, i32, C.POINTER(sz)]
    L.cl_compressed_conv_forward.argtypes = [p, C.POINTER(ConvDesc), p, p, p, i32, i32, i32, p, sz, p]
    L.cl_plan_batches.argtypes = [i32, p, i32, p, p, p, p, i64, i64, C.c_double, p, C.POINTER(C.c_double)]
    L.cl_maxpool_forward.argtypes = [p, p] + [i32] * 6 + [p]
    L.cl_lrn_forward.argtypes = [p, p] + [i32] * 5 + [C.c_float] * 3 + [p]
    L.cl_set_kernel_timing.argtypes = [i32]
    L.cl_last_kernel_ms.argtypes = [C.POINTER(C.c_float), C.POINTER(i32)]
    L.cl_mx_quantize.argtypes = [p, i32, i64, i64, i32, p, p, p]
    L.cl_mx_dequantize.argtypes = [p, p, i64, i32, p, i32, i64, p]
    L.cl_mx_fc_workspace_bytes.argtypes = [C.POINTER(MxMatrix), i32, i32, C.POINTER(sz)]
    L.cl_mx_fc_forward.argtypes = [C.POINTER(MxMatrix), C.POINTER(MxInput), p, p, i32, i32, i32, p, sz, p]
    L.cl_route_experts.argtypes = [p, i32, i64, p, i32, C.POINTER(RouteDesc), p, p, p]
    L.cl_expert_lists_bytes.argtypes = [i32, i32, i32, C.POINTER(sz)]
    L.cl_expert_lists.argtypes = [p, i32, i32, i32, p, sz, p]
    L.cl_mx_experts_workspace_bytes.argtypes = [C.POINTER(MxMatrix), i32, C.POINTER(MxExpertsCall), i32, C.POINTER(sz)]
    L.cl_mx_fc_resolved_form.argtypes = [C.POINTER(MxMatrix), i32, i32, C.POINTER(i32), C.POINTER(i32)]
    L.cl_mx_experts_resolved_form.argtypes = [C.POINTER(MxMatrix), i32, C.POINTER(MxExpertsCall), i32, C.POINTER(i32)]
    L.cl_mx_experts_forward.argtypes = [C.POINTER(MxMatrix), i32, C.POINTER(MxInput), C.POINTER(MxExpertsCall), p, i32, p, sz, p]
    for name in EXPORTS:
        if name not in ("cl_last_error", "cl_layer_group_free"):
            getattr(L, name).restype = i32
    L.cl_layer_group_free.restype = None
    L.cl_layer_group_free.argtypes = [C.c_void_p]
    _lib = L
    return L


def _check(rc):
    if rc != CL_OK:
        raise CLError(rc, lib().cl_last_error().decode())


def _np_ptr(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _dev_ptr(t):
    """Raw device address of a torch CUDA tensor (or None)."""
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous CUDA tensor")
    return C.c_void_p(t.data_ptr())


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _want(t, shape, what):
    """A tensor handed to the library as a raw pointer must be what the kernels
    assume: fp32, contiguous, on the GPU, of exactly this shape."""
    import torch
    if t is None:
        return
    if t.dtype != torch.float32 or tuple(t.shape) != tuple(shape) or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous float32 CUDA tensor of shape {tuple(shape)}, "
                         f"got {t.dtype} {tuple(t.shape)}")


# (a function object of its own: the attribute of ctypes.pythonapi is shared by the whole process)
_new_bytes = C.PYFUNCTYPE(C.py_object, C.c_void_p, C.c_ssize_t)(("PyBytes_FromStringAndSize", C.pythonapi))


class Layer:
    """Owns a cl_layer handle."""

    def __init__(self, handle):
        self._h = C.c_void_p(handle)
        v = HostView()
        _check(lib().cl_layer_host_view(self._h, C.byref(v)))
        self.M, self.K = v.desc.M, v.desc.K
        self._ws_cache = {}

    @property
    def handle(self):
        if not self._h:
            raise ValueError("layer was freed")
        return self._h

    def free(self):
        if self._h:
            lib().cl_layer_free(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    # -- mirrors of the C entry points ------------------------------------- #
    def upload(self):
        _check(lib().cl_layer_upload(self.handle))
        return self

    def stats(self) -> dict:
        s = Stats()
        _check(lib().cl_layer_stats(self.handle, C.byref(s)))
        return {n: getattr(s, n) for n, _ in Stats._fields_}

    def host_view(self) -> dict:
        """numpy copies of the host sections."""
        v = HostView()
        _check(lib().cl_layer_host_view(self.handle, C.byref(v)))
        d = v.desc
        nval, nidx = 1 << d.weight_bits, 1 << d.index_bits

        def arr(ptr, n, dt):
            if n == 0:
                return np.zeros(0, dt)
            return np.ctypeslib.as_array(ptr, shape=(n,)).astype(dt, copy=True)

        nc = int(v.n_chunks)
        meta = np.zeros(nc + 1, dtype=[("sym_off", "<u4"), ("rec_off", "<u4"), ("blk", "<u4"), ("pos0", "<u4")])
        C.memmove(meta.ctypes.data, v.chunk_meta, meta.nbytes)
        return dict(desc={n: getattr(d, n) for n, _ in LayerDesc._fields_},
                    codebook=arr(v.codebook, nval, np.float32), val_len=arr(v.val_len, nval, np.uint8),
                    val_code=arr(v.val_code, nval, np.uint32), idx_len=arr(v.idx_len, nidx, np.uint8),
                    idx_code=arr(v.idx_code, nidx, np.uint32), block_ptr=arr(v.block_ptr, int(v.n_blocks) + 1, np.uint32),
                    panel_chunk=arr(v.panel_chunk, int(v.n_panels) + 1, np.uint32), chunk_meta=meta,
                    records=arr(v.records, int(v.n_records), np.uint64),
                    chunk_nz=arr(v.chunk_nz, nc + 1, np.uint32), max_block_nnz=int(v.max_block_nnz),
                    max_group_blocks=int(v.max_group_blocks),
                    chunk_half=None if not v.group_ptr else
                    arr(v.chunk_half, 2 * nc, np.uint32).reshape(nc, 2) if nc else np.zeros((0, 2), np.uint32),
                    group_ptr=arr(v.group_ptr, int(v.n_blocks) * 34, np.uint32).reshape(int(v.n_blocks), 2, 17) if v.group_ptr else None,
                    n_blocks=int(v.n_blocks), n_chunks=nc, n_records=int(v.n_records), n_entries=int(v.n_entries),
                    n_panels=int(v.n_panels))

    def serialize(self) -> bytes:
        n = C.c_size_t(0)
        _check(lib().cl_layer_serialize(self.handle, None, C.byref(n)))
        buf = _new_bytes(None, n.value)          # written by the library before anything else sees it: no zeroing, no copy
        _check(lib().cl_layer_serialize(self.handle, buf, C.byref(n)))
        return buf


def conv_block_h(out_channels: int, groups: int, block_h: int = 128) -> int:
    """Block height for a convolution layer: with filter groups the library wants
    block_h to divide the filters of a group, so the largest such divisor up to
    block_h (AlexNet conv4, 192 filters per group: 96)."""
    per_group = out_channels // groups
    if groups == 1 or per_group % block_h == 0:
        return block_h
    return max(d for d in range(1, min(block_h, per_group) + 1) if per_group % d == 0)


def compress_layer(W, weight_bits, index_bits, block_h, block_w, codebook=None, max_code_len=0, upload=False) -> Layer:
    W = np.ascontiguousarray(W, np.float32)
    if W.ndim != 2:
        raise ValueError("W must be M x K")
    d = LayerDesc(W.shape[0], W.shape[1], weight_bits, index_bits, block_h, block_w, CHUNK_BITS, max_code_len)
    cb = None if codebook is None else np.ascontiguousarray(codebook, np.float32)
    if cb is not None and cb.size != (1 << weight_bits):
        raise ValueError("codebook must have 2^weight_bits entries")
    out = C.c_void_p()
    _check(lib().cl_compress_layer(C.byref(d), _np_ptr(W), _np_ptr(cb), C.byref(out)))
    layer = Layer(out.value)
    if upload:
        layer.upload()
    return layer


def layer_deserialize(data: bytes) -> Layer:
    out = C.c_void_p()
    _check(lib().cl_layer_deserialize(data, len(data), C.byref(out)))
    return Layer(out.value)


def decode_layer(layer: Layer, want_dense=True):
    """-> (val_sym, idx_sym, block_ptr, dense or None) as torch CUDA tensors."""
    import torch
    st = layer.stats()
    hv = Stats  # noqa: F841 (kept for symmetry with the C names)
    v = HostView()
    _check(lib().cl_layer_host_view(layer.handle, C.byref(v)))
    dev = torch.device("cuda")
    val = torch.empty(st["entries"], dtype=torch.uint8, device=dev)
    idx = torch.empty(st["entries"], dtype=torch.uint8, device=dev)
    bp = torch.empty(st["n_blocks"] + 1, dtype=torch.int32, device=dev)
    dense = torch.empty((v.desc.M, v.desc.K), dtype=torch.float32, device=dev) if want_dense else None
    _check(lib().cl_decode_layer(layer.handle, _dev_ptr(val), _dev_ptr(idx), _dev_ptr(bp), _dev_ptr(dense), _stream()))
    return val, idx, bp, dense


def fc_workspace_bytes(layer: Layer, batch: int, path: int = PATH_AUTO) -> int:
    key = (batch, path)
    if key not in layer._ws_cache:
        n = C.c_size_t(0)
        _check(lib().cl_fc_workspace_bytes(layer.handle, batch, path, C.byref(n)))
        layer._ws_cache[key] = n.value
    return layer._ws_cache[key]


def fc_resolved_path(layer: Layer, batch: int, path: int = PATH_AUTO) -> int:
    """The path cl_compressed_fc_forward takes for (layer, batch, path)."""
    out = C.c_int32(0)
    _check(lib().cl_fc_resolved_path(layer.handle, batch, path, C.byref(out)))
    return out.value


def compressed_fc_forward(layer: Layer, X, bias=None, relu=False, path=PATH_AUTO, out=None, workspace=None):
    """X: (B, K) fp32 CUDA tensor -> Y: (B, M) fp32 CUDA tensor."""
    import torch
    M, K = layer.M, layer.K
    if X.dtype != torch.float32 or X.dim() != 2 or X.shape[1] != K:
        raise ValueError(f"X must be (B, {K}) float32")
    B = X.shape[0]
    _want(X, (B, K), "X")
    _want(bias, (M,), "bias")
    _want(out, (B, M), "out")
    Y = out if out is not None else torch.empty((B, M), dtype=torch.float32, device=X.device)
    need = fc_workspace_bytes(layer, B, path)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=X.device)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().cl_compressed_fc_forward(layer.handle, _dev_ptr(X), _dev_ptr(bias), _dev_ptr(Y), B, int(relu), path,
                                          _dev_ptr(workspace), C.c_size_t(wbytes), _stream()))
    return Y


def compressed_fc_forward_static(layer: Layer, X, out, bias=None, relu=False, path=PATH_AUTO):
    """cl_compressed_fc_forward_static: scratch in the library's static device array; the
    caller brings the output, nothing is allocated here or in the library."""
    B = X.shape[0] if X.dim() == 2 else -1
    _want(X, (B, layer.K), "X")
    _want(bias, (layer.M,), "bias")
    if out is None:
        raise ValueError("the non-allocating call needs the caller's output tensor")
    _want(out, (B, layer.M), "out")
    _check(lib().cl_compressed_fc_forward_static(layer.handle, _dev_ptr(X), _dev_ptr(bias), _dev_ptr(out), B, int(relu), path,
                                                 _stream()))
    return out


def _handles(layers):
    return (C.c_void_p * len(layers))(*[l.handle for l in layers])


def fc_stack_workspace_bytes(layers, batch: int, path: int = PATH_AUTO) -> int:
    n = C.c_size_t(0)
    _check(lib().cl_fc_stack_workspace_bytes(_handles(layers), len(layers), batch, path, C.byref(n)))
    return n.value


def compressed_fc_stack_forward(layers, X, biases=None, relu_hidden=True, relu_last=False, path=PATH_AUTO, out=None,
                                workspace=None):
    """A stack of FC layers in one call: X (B, K_0) fp32 CUDA tensor -> (B, M_last)."""
    import torch
    layers = list(layers)
    if X.dtype != torch.float32 or X.dim() != 2 or X.shape[1] != layers[0].K:
        raise ValueError(f"X must be (B, {layers[0].K}) float32")
    B = X.shape[0]
    _want(X, (B, layers[0].K), "X")
    _want(out, (B, layers[-1].M), "out")
    if biases is not None:
        if len(biases) != len(layers):
            raise ValueError("one bias (or None) per layer")
        for b, l in zip(biases, layers):
            _want(b, (l.M,), "bias")
    Y = out if out is not None else torch.empty((B, layers[-1].M), dtype=torch.float32, device=X.device)
    if workspace is None:
        workspace = torch.empty(max(256, fc_stack_workspace_bytes(layers, B, path)), dtype=torch.uint8, device=X.device)
    bias_ptrs = None
    if biases is not None:
        bias_ptrs = (C.c_void_p * len(layers))(*[None if b is None else _dev_ptr(b).value for b in biases])
    _check(lib().cl_compressed_fc_stack_forward(_handles(layers), len(layers), _dev_ptr(X), bias_ptrs, _dev_ptr(Y), B,
                                                int(relu_hidden), int(relu_last), path, _dev_ptr(workspace),
                                                C.c_size_t(workspace.numel() * workspace.element_size()), _stream()))
    return Y


class LayerGroup:
    """Several uploaded layers of one shape, run in one grid (cl_layer_group_*)."""

    def __init__(self, layers):
        self.layers = list(layers)                       # kept alive: the group holds pointers to them
        h = C.c_void_p()
        _check(lib().cl_layer_group_create(_handles(self.layers), len(self.layers), C.byref(h)))
        self.handle = h

    def free(self):
        if self.handle:
            lib().cl_layer_group_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    def workspace_bytes(self, batch: int) -> int:
        n = C.c_size_t(0)
        _check(lib().cl_fc_group_workspace_bytes(self.handle, batch, C.byref(n)))
        return n.value

    def forward(self, X, bias=None, relu=False, out=None, workspace=None):
        """X: (n, B, K) - one input per layer - or (B, K) shared by all; bias (n, M), (M,) or
        None -> (n, B, M) fp32 CUDA tensor."""
        import torch
        n, L0 = len(self.layers), self.layers[0]
        if X.dtype != torch.float32 or X.dim() not in (2, 3) or X.shape[-1] != L0.K or (X.dim() == 3 and X.shape[0] != n):
            raise ValueError(f"X must be ({n}, B, {L0.K}) or (B, {L0.K}) float32")
        B = X.shape[-2]
        _want(X, tuple(X.shape), "X")
        x_stride = B * L0.K if X.dim() == 3 else 0
        bias_stride = 0
        if bias is not None:
            if bias.dim() == 2:
                _want(bias, (n, L0.M), "bias")
                bias_stride = L0.M
            else:
                _want(bias, (L0.M,), "bias")
        _want(out, (n, B, L0.M), "out")
        Y = out if out is not None else torch.empty((n, B, L0.M), dtype=torch.float32, device=X.device)
        if workspace is None:
            workspace = torch.empty(max(256, self.workspace_bytes(B)), dtype=torch.uint8, device=X.device)
        _check(lib().cl_compressed_fc_group_forward(self.handle, _dev_ptr(X), C.c_size_t(x_stride), _dev_ptr(bias) if bias is not None else None,
                                                    C.c_size_t(bias_stride), _dev_ptr(Y), B, int(relu), _dev_ptr(workspace),
                                                    C.c_size_t(workspace.numel() * workspace.element_size()), _stream()))
        return Y


def conv_workspace_bytes(layer: Layer, conv: dict, batch: int, path: int = PATH_AUTO, compact: bool = False, unsplit: bool = False) -> int:
    """Scratch for the fastest form of the call, for the fastest whose operands are not split beforehand (unsplit), or
    (compact) the least it works with."""
    cd = ConvDesc(conv["C"], conv["H"], conv["W"], conv["R"], conv["S"], conv["stride"], conv["pad"], conv["groups"], conv["OC"])
    n = C.c_size_t(0)
    fn = lib().cl_conv_workspace_bytes_min if compact else lib().cl_conv_workspace_bytes_unsplit if unsplit else lib().cl_conv_workspace_bytes
    _check(fn(layer.handle, C.byref(cd), batch, path, C.byref(n)))
    return n.value


def compressed_conv_forward(layer: Layer, conv: dict, X, bias=None, relu=False, path=PATH_AUTO, out=None, workspace=None):
    """X: (B, C, H, W) fp32 CUDA tensor -> (B, OC, P, Q)."""
    import torch
    cd = ConvDesc(conv["C"], conv["H"], conv["W"], conv["R"], conv["S"], conv["stride"], conv["pad"], conv["groups"], conv["OC"])
    if X.dim() != 4:
        raise ValueError("X must be (B, C, H, W)")
    B = X.shape[0]
    P = (conv["H"] + 2 * conv["pad"] - conv["R"]) // conv["stride"] + 1
    Q = (conv["W"] + 2 * conv["pad"] - conv["S"]) // conv["stride"] + 1
    _want(X, (B, conv["C"], conv["H"], conv["W"]), "X")
    _want(bias, (conv["OC"],), "bias")
    _want(out, (B, conv["OC"], P, Q), "out")
    Y = out if out is not None else torch.empty((B, conv["OC"], P, Q), dtype=torch.float32, device=X.device)
    need = conv_workspace_bytes(layer, conv, B, path)
    if workspace is None and need:
        workspace = torch.empty(need, dtype=torch.uint8, device=X.device)
    wbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().cl_compressed_conv_forward(layer.handle, C.byref(cd), _dev_ptr(X), _dev_ptr(bias), _dev_ptr(Y), B,
                                            int(relu), path, _dev_ptr(workspace), C.c_size_t(wbytes), _stream()))
    return Y


def maxpool_forward(X, size: int, stride: int, out=None):
    """X: (B, C, H, W) fp32 CUDA tensor -> (B, C, P, Q)."""
    import torch
    if X.dtype != torch.float32 or X.dim() != 4 or not X.is_contiguous():
        raise ValueError("X must be a contiguous (B, C, H, W) float32 tensor")
    B, Cc, H, W = X.shape
    P, Q = (H - size) // stride + 1, (W - size) // stride + 1
    _want(out, (B, Cc, max(P, 0), max(Q, 0)), "out")
    if out is not None and out.data_ptr() == X.data_ptr():
        raise ValueError("pooling is not in place")
    Y = out if out is not None else torch.empty((B, Cc, max(P, 0), max(Q, 0)), dtype=torch.float32, device=X.device)
    _check(lib().cl_maxpool_forward(_dev_ptr(X), _dev_ptr(Y), B, Cc, H, W, size, stride, _stream()))
    return Y


def lrn_forward(X, n: int = 5, alpha: float = 1e-4, beta: float = 0.75, k: float = 1.0, out=None):
    """X: (B, C, H, W) fp32 CUDA tensor -> same shape."""
    import torch
    if X.dtype != torch.float32 or X.dim() != 4 or not X.is_contiguous():
        raise ValueError("X must be a contiguous (B, C, H, W) float32 tensor")
    B, Cc, H, W = X.shape
    _want(out, (B, Cc, H, W), "out")
    if out is not None and out.data_ptr() == X.data_ptr():
        raise ValueError("normalisation is not in place: neighbouring channels are read by other workgroups")
    Y = out if out is not None else torch.empty_like(X)
    _check(lib().cl_lrn_forward(_dev_ptr(X), _dev_ptr(Y), B, Cc, H, W, n, float(alpha), float(beta), float(k), _stream()))
    return Y


def plan_batches(time_ms, batch_set, in_bytes_per_image, out_bytes_per_image, ws_bytes, tot_bytes, mem_step_bytes,
                 latency_cap_ms=None):
    """-> (ms_per_image, [batch per layer]) or (inf, None) when nothing is feasible."""
    t = np.ascontiguousarray(time_ms, np.float64)
    f, nb = t.shape
    bs = np.ascontiguousarray(batch_set, np.int32)
    inb = np.ascontiguousarray(in_bytes_per_image, np.int64)
    outb = np.ascontiguousarray(out_bytes_per_image, np.int64)
    ws = np.ascontiguousarray(ws_bytes, np.int64)
    assert bs.size == nb and inb.size == f and outb.size == f and ws.size == f
    plan = np.zeros(f, np.int32)
    ms = C.c_double(0)
    rc = lib().cl_plan_batches(f, _np_ptr(bs), nb, _np_ptr(t), _np_ptr(inb), _np_ptr(outb), _np_ptr(ws), int(tot_bytes),
                               int(mem_step_bytes), float(latency_cap_ms or 0.0), _np_ptr(plan), C.byref(ms))
    if rc == CL_EUNSUPPORTED:
        return float("inf"), None
    _check(rc)
    return ms.value, plan.tolist()


# --------------------------------------------------------------------------- #
# microscaled 4-bit matrices and routed experts
# --------------------------------------------------------------------------- #
# (A call of these takes a few microseconds on the GPU where rows are few: what the host does for it is kept short.)
_types: dict = {}
_current_device = _raw_stream = None


def _start():
    """The library, with what the calls below use of torch at hand."""
    global _current_device, _raw_stream
    if not _types:
        import torch
        L = lib()
        _current_device = torch.cuda.current_device
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
        _types.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
        return L
    return _lib


def _element_type(dtype, what):
    """CL_F32, CL_BF16 or CL_F16."""
    ty = _types.get(dtype)
    if ty is None:
        raise ValueError(f"{what} must be float32, bfloat16 or float16, got {dtype}")
    return ty


def _int32(*sizes):
    """What the library takes in 32 bits: ctypes would cut off what is beyond."""
    for n in sizes:
        if not -1 << 31 <= n < 1 << 31:
            raise ValueError(f"{n} does not fit 32 bits")


def _rows(t, what, cols=None):
    """A matrix whose rows are contiguous, at any distance from each other -> (element type, distance)."""
    ty = _element_type(t.dtype, what)
    shape = t.shape
    if len(shape) != 2 or not t.is_cuda or (cols is not None and shape[1] != cols):
        raise ValueError(f"{what} must be a CUDA matrix{'' if cols is None else f' with rows of {cols}'}, got {tuple(shape)} on {t.device}")
    stride, one = t.stride()
    if one != 1 and shape[1] > 1:
        raise ValueError(f"{what} must have contiguous rows, got strides {t.stride()}")
    return ty, stride if shape[0] > 1 else shape[1]


def _on(device, *tensors):
    """The stream of a call, which runs on the current device: where all its tensors have to be."""
    index = device.index
    if index != _current_device():
        raise ValueError(f"the input is on {device}, the current device is cuda:{_current_device()}")
    for t in tensors:
        if t is not None and t.device != device:
            raise ValueError(f"a tensor is on {t.device}, the input on {device}")
    return _raw_stream(index)


def mx_row_blocks(K: int) -> int:
    """Blocks of a row of K elements: whole groups of four."""
    if K < 1:
        raise ValueError("a row has at least one element")
    return (K + 127) // 128 * 4


class MxTensor:
    """A matrix - or a stack of matrices of one shape, for experts - in blocks of 32 four-bit floats under one scale:
    codes (..., rows, blocks * 16) and scales (..., rows, blocks), uint8, blocks = mx_row_blocks(K)."""

    __slots__ = ("codes", "scales", "K")

    def __init__(self, codes, scales, K):
        kb = mx_row_blocks(K)
        import torch
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or not codes.is_cuda or not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError("codes and scales must be contiguous uint8 CUDA tensors")
        shape = codes.shape
        if len(shape) < 2 or shape[-1] != kb * 16 or scales.shape != shape[:-1] + (kb,) or scales.device != codes.device:
            raise ValueError(f"rows of {K} elements have {kb * 16} bytes of codes and {kb} scales, got {tuple(shape)} and {tuple(scales.shape)}")
        self.codes, self.scales, self.K = codes, scales, K

    @property
    def shape(self):
        return tuple(self.codes.shape[:-1]) + (self.K,)

    @property
    def device(self):
        return self.codes.device


def mx_quantize(X, out: MxTensor | None = None) -> MxTensor:
    """Rows of X ((..., K), float32, bfloat16 or float16; a matrix's rows at any distance) -> MxTensor of the same shape."""
    import torch
    L = _start()
    shape = X.shape
    K, lead = shape[-1], shape[:-1]
    if len(shape) > 2:
        X = X.reshape(-1, K)
    ty, stride = _rows(X, "X")
    _int32(K)
    if out is None:
        kb = mx_row_blocks(K)
        out = MxTensor.__new__(MxTensor)
        out.codes = torch.empty(lead + (kb * 16,), dtype=torch.uint8, device=X.device)
        out.scales = torch.empty(lead + (kb,), dtype=torch.uint8, device=X.device)
        out.K = K
    elif out.shape != lead + (K,):
        raise ValueError(f"out must hold {tuple(lead) + (K,)}, holds {out.shape}")
    stream = _on(X.device, out.codes)
    _check(L.cl_mx_quantize(X.data_ptr(), ty, stride, X.shape[0], K, out.codes.data_ptr(), out.scales.data_ptr(), stream))
    return out


def mx_dequantize(Q: MxTensor, dtype=None, out=None):
    """The values Q stands for, (..., K) of dtype (float32 unless given)."""
    import torch
    L = _start()
    codes = Q.codes
    shape = codes.shape[:-1] + (Q.K,)
    if out is None:
        out = torch.empty(shape, dtype=dtype or torch.float32, device=codes.device)
    elif out.shape != shape or not (out.is_contiguous() or len(shape) == 2) or (dtype is not None and out.dtype != dtype):
        raise ValueError(f"out must be {tuple(shape)}{'' if dtype is None else f' of {dtype}'}, contiguous or a matrix with contiguous rows")
    Y = out if len(shape) == 2 else out.view(-1, Q.K)
    _int32(Q.K)
    ty, stride = _rows(Y, "out", Q.K)
    stream = _on(codes.device, out)
    _check(L.cl_mx_dequantize(codes.data_ptr(), Q.scales.data_ptr(), Y.shape[0], Q.K, out.data_ptr(), ty, stride, stream))
    return out


def _mx_input(X, K):
    """-> (struct, rows, element type of an output that names none)"""
    if isinstance(X, MxTensor):
        if len(X.codes.shape) != 2 or X.K != K:
            raise ValueError(f"X must have rows of {K}, got {X.shape}")
        import torch
        return MxInput(X.codes.data_ptr(), X.scales.data_ptr(), MX4, 0), X.codes.shape[0], torch.float32
    ty, stride = _rows(X, "X", K)
    return MxInput(X.data_ptr(), None, ty, stride), X.shape[0], X.dtype


def _mx_output(out, shape, dtype, device):
    """-> (tensor, element type)"""
    if out is None:
        import torch
        out = torch.empty(shape, dtype=dtype, device=device)
    elif tuple(out.shape) != shape or not out.is_contiguous() or out.dtype != dtype:
        raise ValueError(f"out must be a contiguous {dtype} tensor of shape {shape}, got {out.dtype} {tuple(out.shape)}")
    return out, _element_type(dtype, "out")


def _mx_workspace(workspace, need, device):
    """-> (tensor, address, bytes)"""
    if workspace is None:
        if not need:
            return None, None, 0
        import torch
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
    elif not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _act(act):
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError(f"act must be one of {', '.join(ACTIVATIONS)}, got {act!r}")
    return code


@functools.lru_cache(maxsize=1024)
def _mx_fc_need(M, K, batch, x_type):
    _int32(M, K, batch)
    n = C.c_size_t(0)
    _check(lib().cl_mx_fc_workspace_bytes(MxMatrix(None, None, M, K), batch, x_type, n))
    return n.value


def mx_fc_workspace_bytes(W: MxTensor, batch: int, dtype=None) -> int:
    """Scratch of mx_fc_forward for `batch` rows of dtype (None: an MxTensor), or fewer."""
    _start()
    return _mx_fc_need(W.shape[0], W.K, batch, MX4 if dtype is None else _element_type(dtype, "X"))


def mx_fc_resolved_form(W: MxTensor, batch: int, dtype=None) -> tuple[str, int]:
    """How mx_fc_forward makes `batch` rows of dtype (None: an MxTensor): one of MX_FORMS, and how many sums k is split into."""
    _start()
    _int32(*W.shape, batch)
    form, splits = C.c_int32(0), C.c_int32(0)
    _check(lib().cl_mx_fc_resolved_form(MxMatrix(None, None, W.shape[0], W.K), batch, MX4 if dtype is None else _element_type(dtype, "X"), form, splits))
    return MX_FORMS[form.value], splits.value


def mx_fc_forward(W: MxTensor, X, bias=None, relu=False, act=None, dtype=None, out=None, workspace=None):
    """act(X W^T + bias) with W (M, K) in 4-bit blocks and X (B, K) - float32, bfloat16 or float16, quantised on the way, or an MxTensor.
    act: "none", "relu" (the same as relu=True) or "gated" (rows 2 i and 2 i + 1 of W give gate and value of output i).  The output is of
    dtype, X's own unless given (float32 for an MxTensor)."""
    L = _start()
    codes, K = W.codes, W.K
    if len(codes.shape) != 2:
        raise ValueError(f"W must be a matrix, got {W.shape}")
    M = codes.shape[0]
    if relu and act not in (None, "relu"):
        raise ValueError(f"relu=True and act={act!r}")
    act = _act(act or ("relu" if relu else "none"))
    xs, B, own_dtype = _mx_input(X, K)
    if bias is not None:
        _want(bias, (M,), "bias")
    device = X.device
    Y, y_type = _mx_output(out, (B, M // 2 if act == 2 else M), dtype or (own_dtype if out is None else out.dtype), device)
    stream = _on(device, codes, bias, Y, workspace)
    workspace, ws, ws_bytes = _mx_workspace(workspace, _mx_fc_need(M, K, B, xs.type), device)
    _check(L.cl_mx_fc_forward(MxMatrix(codes.data_ptr(), W.scales.data_ptr(), M, K), xs, None if bias is None else bias.data_ptr(), Y.data_ptr(), y_type, B,
                              act, ws, ws_bytes, stream))
    return Y


def route_experts(logits, k: int, bias=None, score="softmax", groups: int = 1, groups_kept: int | None = None, group_score="max", renormalize=True,
                  scale: float = 1.0):
    """logits (T, E) -> (experts (T, k) int32, weights (T, k) float32): the k experts of each token with the largest scores + bias (within the
    groups_kept best of `groups` runs of experts), and their scores without the bias, divided by their sum if renormalize, times scale.
    -1 and 0 where no expert is left (logits of -inf, the lowest value or NaN mask an expert)."""
    import torch
    L = _start()
    ty, stride = _rows(logits, "logits")
    T, E = logits.shape
    groups_kept = groups if groups_kept is None else groups_kept
    _int32(T, E, k, groups, groups_kept)
    if bias is not None:
        _want(bias, (E,), "bias")
    if score not in SCORES or group_score not in GROUP_SCORES:
        raise ValueError(f"score must be one of {', '.join(SCORES)} and group_score of {', '.join(GROUP_SCORES)}, got {score!r} and {group_score!r}")
    device = logits.device
    stream = _on(device, bias)
    d = RouteDesc(E, k, SCORES[score], groups, groups_kept, GROUP_SCORES[group_score], int(renormalize), scale)
    width = k if 0 < k <= E else 0                           # (other k are refused)
    experts = torch.empty((T, width), dtype=torch.int32, device=device)
    weights = torch.empty((T, width), dtype=torch.float32, device=device)
    _check(L.cl_route_experts(logits.data_ptr(), ty, stride, None if bias is None else bias.data_ptr(), T, d, experts.data_ptr(), weights.data_ptr(), stream))
    return experts, weights


def _want_experts(experts):
    import torch
    if experts.dtype != torch.int32 or experts.dim() != 2 or not experts.is_cuda or not experts.is_contiguous():
        raise ValueError(f"experts must be a contiguous int32 CUDA matrix, got {experts.dtype} {tuple(experts.shape)}")


class ExpertLists:
    """The pairs of a choice of experts in the order of their experts (cl_expert_lists), for several products with one choice."""

    __slots__ = ("buffer", "tokens", "k", "n_experts")

    def __init__(self, buffer, tokens, k, n_experts):
        self.buffer, self.tokens, self.k, self.n_experts = buffer, tokens, k, n_experts

    @property
    def offsets(self):
        """(n_experts + 2) int32: where each expert's pairs begin, where those without one do, and the end."""
        import torch
        return self.buffer[:4 * (self.n_experts + 2)].view(torch.int32)


def expert_lists(experts, n_experts: int) -> ExpertLists:
    """experts (T, k) int32, as route_experts gives them."""
    import torch
    L = _start()
    _want_experts(experts)
    stream = _on(experts.device)
    T, k = experts.shape
    _int32(T, k, n_experts)
    n = C.c_size_t(0)
    _check(L.cl_expert_lists_bytes(T, k, n_experts, n))
    buffer = torch.empty(n.value, dtype=torch.uint8, device=experts.device)
    _check(L.cl_expert_lists(experts.data_ptr(), T, k, n_experts, buffer.data_ptr(), n.value, stream))
    return ExpertLists(buffer, T, k, n_experts)


@functools.lru_cache(maxsize=1024)
def _mx_experts_need(M, K, E, T, k, weighted, lists, act, x_per_pair, x_type):
    _int32(M, K, E, T, k)
    n = C.c_size_t(0)
    call = MxExpertsCall(T, k, None, 256 if weighted else None, None, 256 if lists else None, act, x_per_pair)
    _check(lib().cl_mx_experts_workspace_bytes(MxMatrix(None, None, M, K), E, call, x_type, n))
    return n.value


@functools.lru_cache(maxsize=1024)
def _mx_experts_form(M, K, E, T, k, weighted, lists, x_per_pair, x_type):
    _int32(M, K, E, T, k)
    form = C.c_int32(0)
    call = MxExpertsCall(T, k, None, 256 if weighted else None, None, 256 if lists else None, 0, x_per_pair)
    _check(lib().cl_mx_experts_resolved_form(MxMatrix(None, None, M, K), E, call, x_type, form))
    return MX_FORMS[form.value]


def mx_experts_resolved_form(W: MxTensor, tokens: int, k: int, dtype=None, weighted=True, x_per_pair=False, lists=False) -> str:
    """How mx_experts_forward makes the products of `tokens` rows of dtype (None: an MxTensor) with k experts each: one of MX_FORMS."""
    _start()
    E, M, K = W.shape
    return _mx_experts_form(M, K, E, tokens, k, weighted, lists, int(x_per_pair), MX4 if dtype is None else _element_type(dtype, "X"))


def mx_experts_forward(W: MxTensor, X, experts, weights=None, bias=None, act="none", x_per_pair=False, lists: ExpertLists | None = None, dtype=None,
                       out=None, workspace=None):
    """The products of rows with their experts' matrices: W (E, M, K) in 4-bit blocks, X (T, K) - or (T * k, K) with x_per_pair -, experts (T, k) int32.
    With weights (T, k): (T, M), the weighted sum of each token's k products; without: (T * k, M), one row a pair.  bias (E, M); act as in
    mx_fc_forward, before the sum.  Pairs with an expert outside 0 .. E - 1 give nothing (a row of zeros without weights)."""
    L = _start()
    codes, K = W.codes, W.K
    if len(codes.shape) != 3:
        raise ValueError(f"W must be (experts, rows, K), got {W.shape}")
    E, M, _ = codes.shape
    _want_experts(experts)
    T, k = experts.shape
    act = _act(act)
    xs, rows, own_dtype = _mx_input(X, K)
    if rows != (T * k if x_per_pair else T):
        raise ValueError(f"X must have {T * k if x_per_pair else T} rows, got {rows}")
    if weights is not None:
        _want(weights, (T, k), "weights")
    if bias is not None:
        _want(bias, (E, M), "bias")
    if lists is not None and (lists.tokens, lists.k, lists.n_experts) != (T, k, E):
        raise ValueError(f"lists of {lists.tokens} x {lists.k} of {lists.n_experts} experts, wanted {T} x {k} of {E}")
    device = X.device
    Y, y_type = _mx_output(out, (T if weights is not None else T * k, M // 2 if act == 2 else M), dtype or (own_dtype if out is None else out.dtype), device)
    stream = _on(device, codes, experts, weights, bias, Y, workspace, None if lists is None else lists.buffer)
    need = _mx_experts_need(M, K, E, T, k, weights is not None, lists is not None, act, int(x_per_pair), xs.type)
    workspace, ws, ws_bytes = _mx_workspace(workspace, need, device)
    call = MxExpertsCall(T, k, experts.data_ptr(), None if weights is None else weights.data_ptr(), None if bias is None else bias.data_ptr(),
                         None if lists is None else lists.buffer.data_ptr(), act, int(x_per_pair))
    _check(L.cl_mx_experts_forward(MxMatrix(codes.data_ptr(), W.scales.data_ptr(), M, K), E, xs, call, Y.data_ptr(), y_type, ws, ws_bytes, stream))
    return Y


def set_kernel_timing(enable: bool):
    _check(lib().cl_set_kernel_timing(int(enable)))


def last_kernel_ms():
    """-> (milliseconds, launches) of the main kernel(s) of the last forward call."""
    ms, n = C.c_float(0), C.c_int32(0)
    _check(lib().cl_last_kernel_ms(C.byref(ms), C.byref(n)))
    return ms.value, n.value
