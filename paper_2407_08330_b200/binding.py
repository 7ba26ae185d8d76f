"""ctypes binding of libhdt.so.  Argument marshalling only."""
from __future__ import annotations

import ctypes as C
import functools
import os
import re

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIBPATH = os.path.join(_HERE, "libhdt.so")
_HEADERS = [os.path.join(_HERE, "..", "include", h) for h in ("hdt.h", "hdt_debug.h")]
_lib = None

HDT_F32, HDT_BF16 = 0, 1
HDT_MAX_STAGES = 24
_DTYPES = {torch.float32: HDT_F32, torch.bfloat16: HDT_BF16}


class HdtError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libhdt error {code}: {msg}")
        self.code = code


class _Params(C.Structure):
    _fields_ = [("block_m", C.c_int32), ("max_stages", C.c_int32), ("block_m_upper", C.c_int32),
                ("mask_off", C.c_int32), ("deferred", C.c_int32), ("reserved", C.c_int32 * 3)]


class _StageView(C.Structure):
    _fields_ = [("n", C.c_int32), ("n_blocks", C.c_int32)] + \
               [(nm, C.c_void_p) for nm in ("tok", "par", "rng", "up", "scu", "blocks", "queue", "queue_split")] + \
               [("n_fused", C.c_int32)]


def lib():
    """Load libhdt.so; raises if it has not been built (python -m paper_2407_08330_b200.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIBPATH):
            raise HdtError(-5, f"{_LIBPATH} is missing: build it with `python paper_2407_08330_b200/build.py` "
                               "(there is no fallback path)")
        L = C.CDLL(_LIBPATH)
        L.hdt_index_workspace_bytes.restype = C.c_size_t
        L.hdt_index_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_void_p]
        L.hdt_build_index.restype = C.c_int
        L.hdt_build_index.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                      C.c_void_p, C.c_size_t, C.c_void_p, C.POINTER(C.c_void_p)]
        L.hdt_index_info.restype = C.c_int
        L.hdt_index_info.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        L.hdt_index_export.restype = C.c_int
        L.hdt_index_export.argtypes = [C.c_void_p, C.c_int32, C.POINTER(_StageView)]
        L.hdt_index_destroy.restype = C.c_int
        L.hdt_index_destroy.argtypes = [C.c_void_p]
        L.hdt_attn_workspace_bytes.restype = C.c_size_t
        L.hdt_attn_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
        L.hdt_attn_fwd.restype = C.c_int
        L.hdt_attn_fwd.argtypes = [C.c_void_p] * 6 + [C.c_int32, C.c_int32, C.c_int32, C.c_float,
                                                      C.c_void_p, C.c_size_t, C.c_void_p]
        L.hdt_attn_bwd.restype = C.c_int
        L.hdt_attn_bwd.argtypes = [C.c_void_p] * 10 + [C.c_int32, C.c_int32, C.c_int32, C.c_float,
                                                       C.c_void_p, C.c_size_t, C.c_void_p]
        L.hdt_last_error.restype = C.c_char_p
        L.hdt_launch_count.restype = C.c_int64
        L.hdt_attn_fwd_static_max_bytes.restype = C.c_size_t
        L.hdt_attn_fwd_static.restype = C.c_int
        L.hdt_attn_fwd_static.argtypes = [C.c_void_p] * 6 + [C.c_int32, C.c_int32, C.c_int32, C.c_float, C.c_void_p]
        L.hdt_hpe_workspace_bytes.restype = C.c_size_t
        L.hdt_hpe_workspace_bytes.argtypes = [C.c_void_p, C.c_int32]
        L.hdt_hpe.restype = C.c_int
        L.hdt_hpe.argtypes = [C.c_void_p] * 4 + [C.c_int32] * 4 + [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.hdt_cross_workspace_bytes.restype = C.c_size_t
        L.hdt_cross_workspace_bytes.argtypes = [C.c_int32] * 7
        L.hdt_cross_attn_fwd.restype = C.c_int
        L.hdt_cross_attn_fwd.argtypes = [C.c_void_p] * 3 + [C.c_int32] * 4 + [C.c_void_p] * 5 + [C.c_int32] * 3 + \
                                        [C.c_float, C.c_void_p, C.c_size_t, C.c_void_p]
        L.hdt_cross_attn_bwd.restype = C.c_int
        L.hdt_cross_attn_bwd.argtypes = [C.c_void_p] * 3 + [C.c_int32] * 4 + [C.c_void_p] * 9 + [C.c_int32] * 3 + \
                                        [C.c_float, C.c_void_p, C.c_size_t, C.c_void_p]
        L.hdt_dropout.restype = C.c_int
        L.hdt_dropout.argtypes = [C.c_void_p] * 3 + [C.c_int32, C.c_int64, C.c_int32, C.c_int32, C.c_float, C.c_void_p, C.c_void_p]
        L.hdt_layer_norm_fwd.restype = C.c_int
        L.hdt_layer_norm_fwd.argtypes = [C.c_void_p] * 5 + [C.c_int32, C.c_float, C.c_int64] + [C.c_int32] * 3 + [C.c_float] + [C.c_void_p] * 5
        L.hdt_layer_norm_workspace_bytes.restype = C.c_size_t
        L.hdt_layer_norm_workspace_bytes.argtypes = [C.c_int64, C.c_int32]
        L.hdt_layer_norm_bwd.restype = C.c_int
        L.hdt_layer_norm_bwd.argtypes = [C.c_void_p] * 7 + [C.c_int32, C.c_float, C.c_int64] + [C.c_int32] * 3 + [C.c_void_p] * 5 + [C.c_size_t, C.c_void_p]
        L.hdt_self_workspace_bytes.restype = C.c_size_t
        L.hdt_self_workspace_bytes.argtypes = [C.c_int32] * 10
        L.hdt_self_bucket_borders.restype = C.c_int
        L.hdt_self_bucket_borders.argtypes = [C.c_int32] * 3 + [C.POINTER(C.c_int32)]
        L.hdt_self_attn_fwd.restype = C.c_int
        L.hdt_self_attn_fwd.argtypes = [C.c_void_p] * 3 + [C.c_int32] * 3 + [C.c_void_p] * 4 + [C.c_int32] * 3 + [C.c_void_p] * 2 + [C.c_int32] * 3 + \
                                       [C.c_float, C.c_void_p, C.c_size_t, C.c_void_p]
        L.hdt_self_attn_bwd.restype = C.c_int
        L.hdt_self_attn_bwd.argtypes = [C.c_void_p] * 3 + [C.c_int32] * 3 + [C.c_void_p] * 4 + [C.c_int32] * 3 + [C.c_void_p] * 7 + [C.c_int32] * 3 + \
                                       [C.c_float, C.c_void_p, C.c_size_t, C.c_void_p]
        L.hdt_set_option.restype = C.c_int
        L.hdt_device_status.restype = C.c_int
        L.hdt_device_status.argtypes = [C.c_void_p]
        _lib = L
    return _lib


def declared_symbols():
    """Names of every function the headers under include/ declare."""
    txt = "".join(open(h).read() for h in _HEADERS)
    txt = re.sub(r"/\*.*?\*/", "", txt, flags=re.S)
    return sorted(set(re.findall(r"\b(hdt_[a-z0-9_]+)\s*\(", txt)))


def exported_symbols():
    """(declared, missing): declared functions and those libhdt.so does not export."""
    L = lib()
    names = declared_symbols()
    return names, [n for n in names if not hasattr(L, n)]


def _check(rc):
    if rc != 0:
        raise HdtError(rc, lib().hdt_last_error().decode())


def _stream():
    # the raw handle of the current stream without building a torch.cuda.Stream object (0: the default stream)
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


@functools.lru_cache(maxsize=64)
def _params(block_m, max_stages, block_m_upper=0, directions=7, deferred=False):
    """A parameter block and its address (the library only reads it)."""
    p = _Params()
    p.block_m, p.max_stages, p.block_m_upper = int(block_m), int(max_stages), int(block_m_upper)
    p.mask_off = (~int(directions)) & 7
    p.deferred = 1 if deferred else 0
    return p, C.addressof(p)


@functools.lru_cache(maxsize=256)
def hdt_index_workspace_bytes(batch, total_tokens, block_m=0, max_stages=0, block_m_upper=0) -> int:
    p, addr = _params(block_m, max_stages, block_m_upper)
    return int(lib().hdt_index_workspace_bytes(batch, total_tokens, addr))


class HdtIndex:
    """Owner of a built index: the opaque handle plus the device workspace it points into."""

    def __init__(self, handle, workspace, batch, total_tokens):
        self._h, self._ws = handle, workspace
        self.batch, self.total_tokens = batch, total_tokens
        self._info = None
        self._ws_bytes = {}        # attention workspace sizes, by (heads, head_dim, dtype, bwd)

    def _get_info(self):
        if self._info is None:
            ns, nnz, vis = C.c_int32(), C.c_int64(), C.c_int64()
            _check(lib().hdt_index_info(self._h, C.byref(ns), C.byref(nnz), C.byref(vis)))
            self._info = (ns.value, nnz.value, vis.value)
        return self._info

    @property
    def n_stages(self):
        return self._get_info()[0]

    @property
    def nnz(self):
        return self._get_info()[1]

    @property
    def visited(self):
        return self._get_info()[2]

    @property
    def handle(self):
        return self._h

    def export(self, stage):
        """Device arrays of one stage copied to host numpy arrays (parity tests, inspection)."""
        import numpy as np
        v = _StageView()
        _check(lib().hdt_index_export(self._h, stage, C.byref(v)))
        base = self._ws.data_ptr()

        def arr(ptr, count):
            off = (ptr - base) // 4
            return self._ws.view(torch.int32)[off:off + count].cpu().numpy().copy()
        B = self.batch
        return dict(n=v.n, n_blocks=v.n_blocks, tok=arr(v.tok, v.n), par=arr(v.par, v.n),
                    rng=arr(v.rng, 2 * v.n).reshape(-1, 2), up=arr(v.up, v.n), scu=arr(v.scu, B + 1),
                    blocks=arr(v.blocks, 5 * v.n_blocks).reshape(-1, 5), queue=arr(v.queue, v.n_blocks),
                    queue_split=arr(v.queue_split, v.n_blocks), n_fused=int(v.n_fused))

    def close(self):
        if self._h is not None:
            lib().hdt_index_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def hdt_build_index(level, parent, cu_seqlens, block_m=0, max_stages=0, workspace=None,
                    block_m_upper=0, directions=7, deferred=False) -> HdtIndex:
    """level int8[T], parent int32[T], cu_seqlens int32[B+1]: CUDA tensors.  directions: bits
    1 | 2 | 4 keep the child->parent, sibling<->sibling, parent->child entries (7 = full rule).
    deferred: return once the build is queued; the first call that needs the index's counts on the
    host waits for it (and raises what the build found wrong with the structure arrays)."""
    assert level.is_cuda and parent.is_cuda and cu_seqlens.is_cuda
    assert level.dtype == torch.int8 and parent.dtype == torch.int32 and cu_seqlens.dtype == torch.int32
    level, parent, cu_seqlens = level.contiguous(), parent.contiguous(), cu_seqlens.contiguous()
    T, B = level.numel(), cu_seqlens.numel() - 1
    need = hdt_index_workspace_bytes(B, T, block_m, max_stages, block_m_upper)
    if need == 0:
        raise HdtError(-1, "invalid index parameters")
    _, addr = _params(block_m, max_stages, block_m_upper, directions, deferred)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=level.device)
    h = C.c_void_p()
    rc = (_lib or lib()).hdt_build_index(level.data_ptr(), parent.data_ptr(), cu_seqlens.data_ptr(), B, T, addr,
                                         workspace.data_ptr(), workspace.numel(), _stream(), C.byref(h))
    if rc:
        _check(rc)
    return HdtIndex(h, workspace, B, T)


def hdt_attn_workspace_bytes(index: HdtIndex, heads, head_dim, dtype, bwd) -> int:
    key = (heads, head_dim, dtype, bwd)
    n = index._ws_bytes.get(key)
    if n is None:
        n = int(lib().hdt_attn_workspace_bytes(index.handle, heads, head_dim, _DTYPES[dtype], int(bwd)))
        if n:                      # (0: nothing needed, or an index whose build failed)
            index._ws_bytes[key] = n
    return n


def _ws(index, heads, head_dim, dtype, bwd, device, workspace):
    if workspace is not None:      # the library checks the size itself
        return workspace
    return torch.empty(max(hdt_attn_workspace_bytes(index, heads, head_dim, dtype, bwd), 256), dtype=torch.uint8, device=device)


def hdt_attn_fwd(index: HdtIndex, q, k, v, softmax_scale=0.0, out=None, lse=None, workspace=None):
    """q, k, v: CUDA [T, H, d] float32 or bfloat16, contiguous.  Returns (O, LSE [H, T])."""
    T, H, d = q.shape
    dt = q.dtype
    assert q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and dt == k.dtype == v.dtype
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty((H, T), dtype=torch.float32, device=q.device) if lse is None else lse
    workspace = _ws(index, H, d, dt, 0, q.device, workspace)
    rc = (_lib or lib()).hdt_attn_fwd(index._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), H, d,
                                      _DTYPES[dt], float(softmax_scale), workspace.data_ptr(), workspace.numel(), _stream())
    if rc:
        _check(rc)
    return o, lse


def hdt_attn_bwd(index: HdtIndex, q, k, v, o, lse, d_o, softmax_scale=0.0, dq=None, dk=None, dv=None,
                 workspace=None):
    """Returns (dQ, dK, dV) with the shape and dtype of q."""
    T, H, d = q.shape
    dt = q.dtype
    for t in (q, k, v, o, d_o):
        assert t.is_contiguous() and t.dtype == dt
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(q) if dk is None else dk
    dv = torch.empty_like(q) if dv is None else dv
    workspace = _ws(index, H, d, dt, 1, q.device, workspace)
    rc = (_lib or lib()).hdt_attn_bwd(index._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                                      d_o.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), H, d, _DTYPES[dt],
                                      float(softmax_scale), workspace.data_ptr(), workspace.numel(), _stream())
    if rc:
        _check(rc)
    return dq, dk, dv


def hdt_attn_fwd_static_max_bytes() -> int:
    return int(lib().hdt_attn_fwd_static_max_bytes())


def hdt_attn_fwd_static(index: HdtIndex, q, k, v, softmax_scale=0.0, out=None, lse=None):
    """Forward pass for callers that may not allocate device memory during the call: the scratch
    for the upper stages' partial results is a fixed array inside the library, so nothing is
    allocated here as long as `out` and `lse` are passed in.  Raises HdtError (-4) when the batch
    needs more scratch than hdt_attn_fwd_static_max_bytes().  Calls must not overlap on the GPU."""
    T, H, d = q.shape
    assert q.is_contiguous() and k.is_contiguous() and v.is_contiguous() and q.dtype == k.dtype == v.dtype
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty((H, T), dtype=torch.float32, device=q.device) if lse is None else lse
    _check(lib().hdt_attn_fwd_static(index.handle, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), H, d,
                                     _DTYPES[q.dtype], float(softmax_scale), _stream()))
    return o, lse


def hdt_hpe_workspace_bytes(index: HdtIndex, n_levels=3) -> int:
    L = lib()
    return int(L.hdt_hpe_workspace_bytes(index.handle, n_levels))


def hdt_hpe(index: HdtIndex, level, parent, cu_seqlens, d_model, n_levels=3, dtype=torch.float32, x=None,
            accumulate=False, workspace=None):
    """Hierarchical positional encoding [T, d_model]; with `x` and accumulate=True it is added to x."""
    L = lib()
    T = level.numel()
    if x is None:
        x = torch.empty((T, d_model), dtype=dtype, device=level.device)
    assert x.is_contiguous() and x.shape == (T, d_model)
    if workspace is None:
        workspace = torch.empty(max(hdt_hpe_workspace_bytes(index, n_levels), 256), dtype=torch.uint8, device=level.device)
    _check(L.hdt_hpe(index.handle, level.data_ptr(), parent.data_ptr(), cu_seqlens.data_ptr(), n_levels, d_model, _DTYPES[x.dtype],
                     int(bool(accumulate)), x.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream()))
    return x


@functools.lru_cache(maxsize=256)
def hdt_cross_workspace_bytes(batch, total_tokens, total_q, heads, head_dim, dtype, bwd) -> int:
    L = lib()
    return int(L.hdt_cross_workspace_bytes(batch, total_tokens, total_q, heads, head_dim, _DTYPES[dtype], int(bwd)))


def _cross_common(level, cu_seqlens_k, cu_seqlens_q, q, k):
    assert level.dtype == torch.int8 and cu_seqlens_k.dtype == torch.int32 and cu_seqlens_q.dtype == torch.int32
    Tq, H, d = q.shape
    T, B = k.shape[0], cu_seqlens_k.numel() - 1
    assert cu_seqlens_q.numel() == B + 1 and level.numel() == T
    return B, T, Tq, H, d


def hdt_cross_attn_fwd(level, cu_seqlens_k, cu_seqlens_q, level_mask, q, k, v, softmax_scale=0.0, out=None, lse=None,
                       workspace=None):
    """Decoder rows q [Tq,H,d] attend to the encoder rows of k, v [T,H,d] whose level bit is set in
    level_mask.  Returns (O [Tq,H,d], LSE [H,Tq])."""
    L = lib()
    B, T, Tq, H, d = _cross_common(level, cu_seqlens_k, cu_seqlens_q, q, k)
    assert q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
    if out is None:
        out = torch.empty_like(q)
    if lse is None:
        lse = torch.empty((H, Tq), dtype=torch.float32, device=q.device)
    if workspace is None:
        workspace = torch.empty(hdt_cross_workspace_bytes(B, T, Tq, H, d, q.dtype, 0), dtype=torch.uint8, device=q.device)
    _check(L.hdt_cross_attn_fwd(level.data_ptr(), cu_seqlens_k.data_ptr(), cu_seqlens_q.data_ptr(), B, T, Tq, int(level_mask), q.data_ptr(),
                                k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), H, d, _DTYPES[q.dtype], float(softmax_scale),
                                workspace.data_ptr(), workspace.numel(), _stream()))
    return out, lse


def hdt_cross_attn_bwd(level, cu_seqlens_k, cu_seqlens_q, level_mask, q, k, v, o, lse, do, softmax_scale=0.0, dq=None,
                       dk=None, dv=None, workspace=None):
    """Gradients (dQ [Tq,H,d], dK, dV [T,H,d]) of hdt_cross_attn_fwd."""
    L = lib()
    B, T, Tq, H, d = _cross_common(level, cu_seqlens_k, cu_seqlens_q, q, k)
    assert all(x.is_contiguous() for x in (q, k, v, o, do))
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    if workspace is None:
        workspace = torch.empty(hdt_cross_workspace_bytes(B, T, Tq, H, d, q.dtype, 1), dtype=torch.uint8, device=q.device)
    _check(L.hdt_cross_attn_bwd(level.data_ptr(), cu_seqlens_k.data_ptr(), cu_seqlens_q.data_ptr(), B, T, Tq, int(level_mask), q.data_ptr(),
                                k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), do.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), H, d,
                                _DTYPES[q.dtype], float(softmax_scale), workspace.data_ptr(), workspace.numel(), _stream()))
    return dq, dk, dv


def _fit(*sizes):
    """The C interface's sizes have 32 bits (ctypes takes others modulo 2^32)."""
    return max(sizes) < 2 ** 31 and min(sizes) >= -2 ** 31


def _sizes(*sizes):
    if not _fit(*sizes):
        raise HdtError(-3, f"sizes must fit 32 bits: {sizes}")


def _here(*tensors):
    """The tensors of a call are contiguous and on the current device, whose current stream the call goes to."""
    dev = torch._C._cuda_getDevice()
    for t in tensors:
        if t is not None and (t.get_device() != dev or not t.is_contiguous()):      # (get_device: -1 on the CPU)
            raise HdtError(-1, "every tensor must be contiguous and on the current CUDA device")


def _rng(rng, p):
    if rng is None:
        return None
    if rng.dtype != torch.int64 or rng.numel() != 2:
        raise HdtError(-1, "rng must be int64 [2]: seed, offset")
    _here(rng)
    return rng.data_ptr()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _like(t, *others):
    for x in others:
        if x is not None and (x.shape != t.shape or x.dtype != t.dtype):
            raise HdtError(-1, "tensors of one call must have the same shape and type")


def _rows(x):
    """(rows, columns, type): all dimensions but the last are rows."""
    if x.dim() < 1 or x.dtype not in _DTYPES:
        raise HdtError(-3, "rows must be float32 or bfloat16")
    if x.shape[-1] >= 2 ** 31:
        raise HdtError(-3, "sizes must fit 32 bits")
    return (x.numel() // x.shape[-1] if x.shape[-1] else 0), x.shape[-1], _DTYPES[x.dtype]


def hdt_dropout(x, p, rng, site=0, residual=None, out=None):
    """residual + D o x for x [..., cols], D the scaled keep mask of (rng, site): rng is a CUDA int64 tensor [2] = seed,
    offset.  The gradient with respect to x is the same call on the gradient of the result, without a residual."""
    rows, cols, dt = _rows(x)
    if rng is None:
        raise HdtError(-1, "hdt_dropout: p > 0 needs the generator's state")
    _here(x, residual, out)
    _like(x, residual, out)
    y = torch.empty_like(x) if out is None else out
    rc = (_lib or lib()).hdt_dropout(x.data_ptr(), _ptr(residual), _rng(rng, p), int(site), rows, cols, dt, float(p), y.data_ptr(), _stream())
    if rc:
        _check(rc)
    return y


def _norm_weights(cols, *weights):
    for w in weights:
        if w.numel() != cols or w.dtype not in _DTYPES or w.dtype != weights[0].dtype:
            raise HdtError(-1, "weight and bias must have one element per column and one type")


def hdt_layer_norm_fwd(x, weight, bias, eps=1e-5, residual=None, p=0.0, rng=None, site=0, h=None, out=None, mean=None, rstd=None):
    """h = residual + D o x, y = layer norm of h over the last dimension.  Returns (y, h, mean, rstd); h is x itself
    without a residual and without dropout."""
    rows, cols, dt = _rows(x)
    _here(x, residual, out, h, mean, rstd, weight, bias)
    _like(x, residual, out, h)
    _norm_weights(cols, weight, bias)
    for t in (mean, rstd):
        if t is not None and (t.numel() != rows or t.dtype != torch.float32):
            raise HdtError(-1, "mean and rstd must be float32, one element per row")
    y = torch.empty_like(x) if out is None else out
    if h is None and (residual is not None or p > 0):
        h = torch.empty_like(x)
    if mean is None:
        mean = x.new_empty(x.shape[:-1], dtype=torch.float32)
    if rstd is None:
        rstd = torch.empty_like(mean)
    rc = (_lib or lib()).hdt_layer_norm_fwd(x.data_ptr(), _ptr(residual), weight.data_ptr(), bias.data_ptr(), _rng(rng, p), int(site), float(p), rows, cols, dt,
                                            _DTYPES[weight.dtype], float(eps), _ptr(h), y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), _stream())
    if rc:
        _check(rc)
    return y, (x if h is None else h), mean, rstd


@functools.lru_cache(maxsize=256)
def hdt_layer_norm_workspace_bytes(rows, cols) -> int:
    return 0 if not _fit(cols, 0) else int(lib().hdt_layer_norm_workspace_bytes(rows, cols))


def hdt_layer_norm_bwd(d_y, h, mean, rstd, weight, d_h=None, p=0.0, rng=None, site=0, d_residual=None, d_x=None, d_weight=None, d_bias=None,
                       workspace=None):
    """Gradients (d_x, d_residual, d_weight, d_bias) of hdt_layer_norm_fwd; d_h is the gradient that h gets from elsewhere.
    Without dropout d_x and d_residual are one tensor, or, where d_x is given, two with the same values."""
    rows, cols, dt = _rows(h)
    _here(d_y, d_h, h, d_residual, d_x, mean, rstd, weight, d_weight, d_bias, workspace)
    _like(h, d_y, d_h, d_residual, d_x)
    _norm_weights(cols, weight, *(t for t in (d_weight, d_bias) if t is not None))
    d_residual = torch.empty_like(h) if d_residual is None else d_residual
    if p > 0 and d_x is None:
        d_x = torch.empty_like(h)
    d_weight = torch.empty_like(weight) if d_weight is None else d_weight
    d_bias = torch.empty_like(weight) if d_bias is None else d_bias
    if workspace is None:
        workspace = h.new_empty(max(hdt_layer_norm_workspace_bytes(rows, cols), 256), dtype=torch.uint8)
    if mean.numel() != rows or rstd.numel() != rows or mean.dtype != torch.float32 or rstd.dtype != torch.float32:
        raise HdtError(-1, "mean and rstd must be float32, one element per row")
    rc = (_lib or lib()).hdt_layer_norm_bwd(d_y.data_ptr(), _ptr(d_h), h.data_ptr(), mean.data_ptr(), rstd.data_ptr(), weight.data_ptr(), _rng(rng, p), int(site),
                                            float(p), rows, cols, dt, _DTYPES[weight.dtype], d_residual.data_ptr(), _ptr(d_x), d_weight.data_ptr(), d_bias.data_ptr(),
                                            workspace.data_ptr(), workspace.numel(), _stream())
    if rc:
        _check(rc)
    return (d_residual if d_x is None else d_x), d_residual, d_weight, d_bias


@functools.lru_cache(maxsize=256)
def hdt_self_workspace_bytes(batch, total_q, total_k, heads, head_dim, num_buckets, max_distance, causal, dtype, bwd) -> int:
    if not _fit(batch, total_q, total_k, heads, head_dim, num_buckets, max_distance):
        return 0
    return int(lib().hdt_self_workspace_bytes(batch, total_q, total_k, heads, head_dim, num_buckets, max_distance, int(causal), _DTYPES[dtype], int(bwd)))


def hdt_self_bucket_borders(num_buckets, max_distance, causal=True):
    """Smallest distance of every bucket of one direction (a list of num_buckets, or of half of them if not causal)."""
    _sizes(num_buckets, max_distance)
    first = (C.c_int32 * max(1, num_buckets))()
    _check(lib().hdt_self_bucket_borders(int(num_buckets), int(max_distance), int(bool(causal)), first))
    return list(first)[:num_buckets if causal else num_buckets // 2]


def _self_common(cu_q, cu_k, seqlens_k, q, k, v, bias, max_distance):
    if q.dim() != 3 or q.dtype not in _DTYPES or k.shape[1:] != q.shape[1:] or k.dtype != q.dtype:
        raise HdtError(-1, "q, k and v must be [rows, heads, head_dim], float32 or bfloat16 alike")
    _like(k, v)
    B = cu_q.numel() - 1
    for t, n in ((cu_q, B + 1), (cu_k, B + 1), (seqlens_k, B)):
        if t is not None and (t.dtype != torch.int32 or t.numel() != n):
            raise HdtError(-1, "offsets must be int32 [batch + 1], lengths int32 [batch]")
    if bias is not None and (bias.dim() != 2 or bias.shape[1] != q.shape[1] or bias.dtype != q.dtype):
        raise HdtError(-1, "bias must be [num_buckets, heads] of q's type")
    sizes = B, q.shape[0], k.shape[0], q.shape[1], q.shape[2], (0 if bias is None else bias.shape[0])
    _sizes(*sizes, max_distance)
    return sizes


def hdt_self_attn_fwd(cu_seqlens_q, cu_seqlens_k, q, k, v, bias=None, max_distance=128, causal=True, softmax_scale=0.0, seqlens_k=None, out=None,
                      lse=None, workspace=None):
    """Self-attention of packed documents with a bias [num_buckets, heads] by relative position: q [Tq,H,d] (the last rows
    of every document), k, v [Tk,H,d]; seqlens_k [batch] where a document's part of k and v has room behind its keys (a
    cache).  Returns (O [Tq,H,d], LSE [H,Tq]).  Rows of no document are not written: where there are such rows, give `out` and `lse`
    what they are to hold."""
    B, Tq, Tk, H, d, n = _self_common(cu_seqlens_q, cu_seqlens_k, seqlens_k, q, k, v, bias, max_distance)
    _here(cu_seqlens_q, cu_seqlens_k, seqlens_k, q, k, v, bias, out, lse, workspace)
    _like(q, out)
    if lse is not None and (lse.shape != (H, Tq) or lse.dtype != torch.float32):
        raise HdtError(-1, "lse must be float32 [heads, rows of q]")
    out = torch.empty_like(q) if out is None else out
    lse = q.new_empty((H, Tq), dtype=torch.float32) if lse is None else lse
    if workspace is None:
        workspace = q.new_empty(max(256, hdt_self_workspace_bytes(B, Tq, Tk, H, d, n, max_distance, bool(causal), q.dtype, False)), dtype=torch.uint8)
    rc = (_lib or lib()).hdt_self_attn_fwd(cu_seqlens_q.data_ptr(), cu_seqlens_k.data_ptr(), _ptr(seqlens_k), B, Tq, Tk, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                           _ptr(bias), n, int(max_distance), int(bool(causal)), out.data_ptr(), lse.data_ptr(), H, d, _DTYPES[q.dtype],
                                           float(softmax_scale), workspace.data_ptr(), workspace.numel(), _stream())
    if rc:
        _check(rc)
    return out, lse


def hdt_self_attn_bwd(cu_seqlens_q, cu_seqlens_k, q, k, v, o, lse, d_o, bias=None, max_distance=128, causal=True, softmax_scale=0.0, seqlens_k=None,
                      dq=None, dk=None, dv=None, d_bias=None, workspace=None):
    """Gradients (dQ, dK, dV, dBias) of hdt_self_attn_fwd; dBias is None without a bias.  Rows of no document (and keys behind seqlens_k)
    are not written: where there are such rows, give dq, dk and dv zeros."""
    B, Tq, Tk, H, d, n = _self_common(cu_seqlens_q, cu_seqlens_k, seqlens_k, q, k, v, bias, max_distance)
    _here(cu_seqlens_q, cu_seqlens_k, seqlens_k, q, k, v, bias, o, lse, d_o, dq, dk, dv, d_bias, workspace)
    _like(q, o, d_o, dq)
    _like(k, dk, dv)
    if bias is not None:
        _like(bias, d_bias)
    if lse.shape != (H, Tq) or lse.dtype != torch.float32:
        raise HdtError(-1, "lse must be float32 [heads, rows of q]")
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(k) if dv is None else dv
    if bias is not None and d_bias is None:
        d_bias = torch.empty_like(bias)
    if workspace is None:
        workspace = q.new_empty(max(256, hdt_self_workspace_bytes(B, Tq, Tk, H, d, n, max_distance, bool(causal), q.dtype, True)), dtype=torch.uint8)
    rc = (_lib or lib()).hdt_self_attn_bwd(cu_seqlens_q.data_ptr(), cu_seqlens_k.data_ptr(), _ptr(seqlens_k), B, Tq, Tk, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                           _ptr(bias), n, int(max_distance), int(bool(causal)), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(), dq.data_ptr(),
                                           dk.data_ptr(), dv.data_ptr(), _ptr(d_bias), H, d, _DTYPES[q.dtype], float(softmax_scale), workspace.data_ptr(),
                                           workspace.numel(), _stream())
    if rc:
        _check(rc)
    return dq, dk, dv, (None if bias is None else d_bias)


def hdt_set_option(name: str, value: int) -> None:
    _check(lib().hdt_set_option(C.c_char_p(name.encode()), C.c_int32(int(value))))


def hdt_device_status() -> None:
    """Wait for the current stream and raise if a kernel recorded a device-side failure."""
    _check(lib().hdt_device_status(_stream()))


def hdt_launch_count() -> int:
    return int(lib().hdt_launch_count())
