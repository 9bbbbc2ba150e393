"""Thin ctypes binding of libznni.so (declared in include/znni.h): argument marshalling only.

PyTorch is used for device memory and streams; every step of the layer runs in the library's HIP kernels.
There is no fallback: if the compiled library is missing, loading raises.
"""
import ctypes
import functools
import os
import struct

import torch  # imported before the library so both share one HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libznni.so")

OK = 0
RELU = 1
MAC_REFERENCE = 2
MAC_SINGLE = 4
MAC_BATCH = 8
MAC_XDIRECT = 16
MAC_XBLOCK = 32
KEEP_KERNELS = 64
PASSES_REFERENCE = 128
STAGES = ("kernel_prep", "fwd_z", "fwd_y", "fwd_x", "mac", "inv_x", "inv_y", "inv_z")
EXPORTS = ("znni_version", "znni_status_string", "znni_fft_size", "znni_conv3d_fft_workspace",
           "znni_conv3d_fft", "znni_conv3d_fft_profile", "znni_conv3d_fft_workspace_v", "znni_conv3d_fft_v",
           "znni_conv3d_fft_profile_v", "znni_conv3d_fft_static_v", "znni_conv3d_fft_stage_work_v", "znni_conv3d_fft_call_work_v", "znni_conv3d_fft_sublayers_v", "znni_conv3d_fft_budget_v", "znni_conv3d_direct_workspace_v", "znni_conv3d_direct_v", "znni_conv3d_choose_v", "znni_conv3d_workspace_v", "znni_conv3d_v", "znni_mpf", "znni_maxpool",
           "znni_copy_probe", "znni_rope_axes", "znni_attn_window_workspace", "znni_attn_window", "znni_kv8_append",
           "znni_kv8_attn_workspace", "znni_kv8_attn", "znni_attn_window_stats", "znni_attn_window_backward_workspace",
           "znni_attn_window_backward", "znni_linear_workspace", "znni_linear", "znni_linear_backward_workspace",
           "znni_linear_backward", "znni_block_norm", "znni_block_norm_backward_workspace", "znni_block_norm_backward")

F32, BF16, F16 = 0, 1, 2
ALL = 2147483647
KV8_PAGE = 64
ROPE_NEIGHBOURS = 1
_PAIRINGS = {"halves": 0, "neighbours": ROPE_NEIGHBOURS}
_ACTIVATIONS = {None: 0, "relu": 1, "gelu": 2, "silu": 3}
LINEAR_DX, LINEAR_DW, LINEAR_DBIAS = 1, 2, 4
NORM_POST, NORM_PRE, NORM_CENTRED, NORM_GATE_SHARED = 1, 2, 4, 8

_lib = None


class ZnniError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"znni status {status}: {message}")
        self.status = status


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is not built; run `python -m paper_1606_05688_amd.build` "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        i, u, vp, sz = ctypes.c_int, ctypes.c_uint, ctypes.c_void_p, ctypes.c_size_t
        L.znni_version.restype = i
        L.znni_status_string.restype = ctypes.c_char_p
        L.znni_status_string.argtypes = [i]
        L.znni_fft_size.restype = i
        L.znni_fft_size.argtypes = [i]
        L.znni_conv3d_fft_workspace.restype = i
        L.znni_conv3d_fft_workspace.argtypes = [i, i, i, i, i, ctypes.POINTER(sz)]
        L.znni_conv3d_fft.restype = i
        L.znni_conv3d_fft.argtypes = [i, i, i, i, i, vp, vp, vp, vp, u, vp, sz, vp]
        L.znni_conv3d_fft_profile.restype = i
        L.znni_conv3d_fft_profile.argtypes = [i, i, i, i, i, vp, vp, vp, vp, u, vp, sz, vp,
                                              ctypes.POINTER(ctypes.c_float)]
        i3 = ctypes.POINTER(ctypes.c_int)
        L.znni_conv3d_fft_workspace_v.restype = i
        L.znni_conv3d_fft_workspace_v.argtypes = [i, i, i, i3, i3, ctypes.POINTER(sz)]
        L.znni_conv3d_fft_v.restype = i
        L.znni_conv3d_fft_v.argtypes = [i, i, i, i3, i3, vp, vp, vp, vp, u, vp, sz, vp]
        L.znni_conv3d_fft_static_v.restype = i
        L.znni_conv3d_fft_static_v.argtypes = [i, i, i, i3, i3, vp, vp, vp, vp, u, vp]
        for fn in (L.znni_conv3d_fft_stage_work_v, L.znni_conv3d_fft_call_work_v):
            fn.restype = i
            fn.argtypes = [i, i, i, i3, i3, u, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
        L.znni_conv3d_fft_profile_v.restype = i
        L.znni_conv3d_fft_profile_v.argtypes = [i, i, i, i3, i3, vp, vp, vp, vp, u, vp, sz, vp,
                                                ctypes.POINTER(ctypes.c_float)]
        L.znni_conv3d_fft_sublayers_v.restype = i
        L.znni_conv3d_fft_sublayers_v.argtypes = [i, i, i, i3, i3, sz, i3, ctypes.POINTER(sz)]
        L.znni_conv3d_fft_budget_v.restype = i
        L.znni_conv3d_fft_budget_v.argtypes = [i, i, i, i3, i3, vp, vp, vp, vp, u, vp, sz, vp]
        L.znni_conv3d_direct_workspace_v.restype = i
        L.znni_conv3d_direct_workspace_v.argtypes = [i, i, i, i3, i3, ctypes.POINTER(sz)]
        L.znni_conv3d_direct_v.restype = i
        L.znni_conv3d_direct_v.argtypes = [i, i, i, i3, i3, vp, vp, vp, vp, u, vp, sz, vp]
        L.znni_conv3d_choose_v.restype = i
        L.znni_conv3d_choose_v.argtypes = [i, i, i, i3, i3, i3, ctypes.POINTER(ctypes.c_float)]
        L.znni_conv3d_workspace_v.restype = i
        L.znni_conv3d_workspace_v.argtypes = [i, i, i, i3, i3, ctypes.POINTER(sz)]
        L.znni_conv3d_v.restype = i
        L.znni_conv3d_v.argtypes = [i, i, i, i3, i3, vp, vp, vp, vp, u, vp, sz, vp]
        for fn in (L.znni_mpf, L.znni_maxpool):
            fn.restype = i
            fn.argtypes = [i, i, i3, i3, vp, vp, vp]
        hp = ip = vp                     # znni_heads *, int *: bytes that hold them
        L.znni_rope_axes.restype = i
        L.znni_rope_axes.argtypes = [i, i, i, i, i, hp, hp, vp, vp, i, ip, hp, hp, u, vp]
        L.znni_attn_window_workspace.restype = i
        L.znni_attn_window_workspace.argtypes = [i] * 10 + [ctypes.POINTER(sz)]
        L.znni_attn_window.restype = i
        L.znni_attn_window.argtypes = [i, i, i, i, i, hp, hp, hp, vp, vp, i, i, i, i, i, ctypes.c_float, hp, vp, sz, vp]
        L.znni_kv8_append.restype = i
        L.znni_kv8_append.argtypes = [i, i, i, i, hp, hp, vp, vp, i, vp, vp, vp, i, vp, i, vp]
        L.znni_kv8_attn_workspace.restype = i
        L.znni_kv8_attn_workspace.argtypes = [i] * 9 + [ctypes.POINTER(sz)]
        L.znni_kv8_attn.restype = i
        L.znni_kv8_attn.argtypes = [i, i, i, i, i, i, hp, vp, vp, vp, i, vp, i, vp, i, i, i, ctypes.c_float, hp, vp, sz, vp]
        L.znni_attn_window_stats.restype = i
        L.znni_attn_window_stats.argtypes = [i, i, i, i, i, hp, hp, hp, vp, vp, i, i, i, i, i, ctypes.c_float, hp, vp, vp, sz, vp]
        L.znni_attn_window_backward_workspace.restype = i
        L.znni_attn_window_backward_workspace.argtypes = [i] * 10 + [ctypes.POINTER(sz)]
        L.znni_attn_window_backward.restype = i
        L.znni_attn_window_backward.argtypes = [i, i, i, i, i, hp, hp, hp, hp, vp, hp, vp, vp, i, i, i, i, i, ctypes.c_float, hp, hp, hp, vp, sz, vp]
        rp, szp, fl = vp, ctypes.POINTER(sz), ctypes.c_float               # znni_rows *: bytes that hold one
        L.znni_linear_workspace.restype = i
        L.znni_linear_workspace.argtypes = [i, i, i, i, szp]
        L.znni_linear.restype = i
        L.znni_linear.argtypes = [i, i, i, i, rp, rp, vp, i, rp, rp, rp, vp, sz, vp]
        L.znni_linear_backward_workspace.restype = i
        L.znni_linear_backward_workspace.argtypes = [i, i, i, i, i, u, szp]
        L.znni_linear_backward.restype = i
        L.znni_linear_backward.argtypes = [i, i, i, i, rp, rp, rp, rp, i, rp, rp, vp, vp, sz, vp]
        L.znni_block_norm.restype = i
        L.znni_block_norm.argtypes = [i, i, i, rp, rp, rp, vp, vp, fl, fl, u, rp, rp, vp]
        L.znni_block_norm_backward_workspace.restype = i
        L.znni_block_norm_backward_workspace.argtypes = [i, i, i, u, szp]
        L.znni_block_norm_backward.restype = i
        L.znni_block_norm_backward.argtypes = [i, i, i, rp, rp, rp, rp, rp, vp, vp, fl, fl, u, rp, rp, rp, vp, vp, vp, sz, vp]
        L.znni_copy_probe.restype = i
        L.znni_copy_probe.argtypes = [vp, vp, sz, vp]
        _lib = L
    return _lib


def _check(status):
    if status != OK:
        raise ZnniError(status, lib().znni_status_string(status).decode())


def znni_version():
    return int(lib().znni_version())


def znni_fft_size(n):
    return int(lib().znni_fft_size(int(n)))


def _triple(v):
    """An edge length or a sequence <x, y, z> -> ctypes int[3]."""
    t = (int(v),) * 3 if isinstance(v, int) else tuple(int(e) for e in v)
    assert len(t) == 3, "a size is one edge length or three (x, y, z)"
    return (ctypes.c_int * 3)(*t)


def znni_conv3d_fft_workspace(S, f, fo, n, k):
    """Workspace bytes for a layer; n and k are an edge length (cubic call) or (x, y, z) triples (general call)."""
    b = ctypes.c_size_t(0)
    if isinstance(n, int) and isinstance(k, int):
        _check(lib().znni_conv3d_fft_workspace(int(S), int(f), int(fo), n, k, ctypes.byref(b)))
    else:
        _check(lib().znni_conv3d_fft_workspace_v(int(S), int(f), int(fo), _triple(n), _triple(k), ctypes.byref(b)))
    return int(b.value)


def alloc_workspace(S, f, fo, n, k, device="cuda"):
    """A torch byte tensor large enough for the layer (torch allocations are at least 256-byte aligned)."""
    return torch.empty(znni_conv3d_fft_workspace(S, f, fo, n, k), dtype=torch.uint8, device=device)


def _flags(relu, mac_reference, keep_kernels=False):
    """mac_reference: False/True, or one of the strings 'single' / 'batch' / 'xdirect' / 'xblock' to force a
    multiply-accumulate form, or 'generic_passes' for the diagnostic that runs the generic transform passes."""
    m = {False: 0, None: 0, True: MAC_REFERENCE, "reference": MAC_REFERENCE, "single": MAC_SINGLE,
         "batch": MAC_BATCH, "xdirect": MAC_XDIRECT, "xblock": MAC_XBLOCK,
         "generic_passes": PASSES_REFERENCE}[mac_reference]
    return (RELU if relu else 0) | m | (KEEP_KERNELS if keep_kernels else 0)


def _marshal(inp, w, bias, out, workspace):
    assert inp.is_cuda and inp.dtype == torch.float32 and inp.is_contiguous() and inp.dim() == 5
    assert w.is_cuda and w.dtype == torch.float32 and w.is_contiguous() and w.dim() == 5
    S, f = inp.shape[0], inp.shape[1]
    n = tuple(int(e) for e in inp.shape[2:])
    fo = w.shape[0]
    k = tuple(int(e) for e in w.shape[2:])
    assert w.shape[1] == f, "kernel bank must be [f', f, kx, ky, kz]"
    oshape = (S, fo) + tuple(a - b + 1 for a, b in zip(n, k))
    if bias is not None:
        assert bias.is_cuda and bias.dtype == torch.float32 and bias.is_contiguous() and bias.shape == (fo,)
    if out is None:
        out = torch.empty([max(e, 0) for e in oshape], dtype=torch.float32, device=inp.device)
    else:
        assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous()
        assert tuple(out.shape) == oshape
    if workspace is None:
        workspace = alloc_workspace(S, f, fo, n, k, inp.device)
    assert workspace.is_cuda and workspace.dtype == torch.uint8 and workspace.is_contiguous()
    return S, f, fo, n, k, out, workspace


def _cubic(n, k):
    return n[0] == n[1] == n[2] and k[0] == k[1] == k[2]


def znni_conv3d_fft(inp, w, bias=None, relu=False, out=None, workspace=None, stream=None,
                    mac_reference=False, keep_kernels=False):
    """out[S,f',n-k+1 per axis] = act(bias + valid 3D convolution of inp[S,f,nx,ny,nz] with w[f',f,kx,ky,kz]).

    Cubic shapes go through znni_conv3d_fft, all others through znni_conv3d_fft_v.
    Asynchronous on `stream` (a torch.cuda.Stream; default: torch's current stream).
    keep_kernels: the workspace (which must then be passed) still holds this w's stored transforms."""
    assert not keep_kernels or workspace is not None
    S, f, fo, n, k, out, workspace = _marshal(inp, w, bias, out, workspace)
    st = stream if stream is not None else torch.cuda.current_stream(inp.device)
    tail = (inp.data_ptr(), w.data_ptr(), bias.data_ptr() if bias is not None else None, out.data_ptr(),
            _flags(relu, mac_reference, keep_kernels), workspace.data_ptr(), workspace.numel(), st.cuda_stream)
    if _cubic(n, k):
        _check(lib().znni_conv3d_fft(S, f, fo, n[0], k[0], *tail))
    else:
        _check(lib().znni_conv3d_fft_v(S, f, fo, _triple(n), _triple(k), *tail))
    return out


STATIC_SCRATCH_BYTES = 64 << 20


def znni_conv3d_fft_static(inp, w, bias=None, relu=False, out=None, stream=None, mac_reference=False):
    """znni_conv3d_fft on the library's own fixed scratch array instead of a caller's workspace (`out` should be
    passed by callers that must not allocate; without it torch allocates the result)."""
    S, f, fo, n, k, out, _ = _marshal(inp, w, bias, out, inp.new_empty(0, dtype=torch.uint8))
    st = stream if stream is not None else torch.cuda.current_stream(inp.device)
    _check(lib().znni_conv3d_fft_static_v(S, f, fo, _triple(n), _triple(k), inp.data_ptr(), w.data_ptr(),
                                          bias.data_ptr() if bias is not None else None, out.data_ptr(),
                                          _flags(relu, mac_reference), st.cuda_stream))
    return out


def znni_conv3d_fft_profile(inp, w, bias=None, relu=False, out=None, workspace=None, stream=None,
                            mac_reference=False, keep_kernels=False):
    """Same call with per-stage HIP-event timing; returns (out, {stage: milliseconds}).  Synchronises."""
    S, f, fo, n, k, out, workspace = _marshal(inp, w, bias, out, workspace)
    st = stream if stream is not None else torch.cuda.current_stream(inp.device)
    ms = (ctypes.c_float * len(STAGES))()
    tail = (inp.data_ptr(), w.data_ptr(), bias.data_ptr() if bias is not None else None, out.data_ptr(),
            _flags(relu, mac_reference, keep_kernels), workspace.data_ptr(), workspace.numel(), st.cuda_stream, ms)
    if _cubic(n, k):
        _check(lib().znni_conv3d_fft_profile(S, f, fo, n[0], k[0], *tail))
    else:
        _check(lib().znni_conv3d_fft_profile_v(S, f, fo, _triple(n), _triple(k), *tail))
    return out, {name: float(ms[i]) for i, name in enumerate(STAGES)}


def znni_conv3d_fft_stage_work(S, f, fo, n, k, relu=False, mac_reference=False):
    """({stage: bytes the stage must move}, {stage: flops of its contraction}) by the route a call would take through whole planes."""
    return _work(lib().znni_conv3d_fft_stage_work_v, S, f, fo, n, k, _flags(relu, mac_reference))


def znni_conv3d_fft_call_work(S, f, fo, n, k, relu=False, mac_reference=False, keep_kernels=False):
    """The same for the kernels the call runs, planes cut into tiles included."""
    return _work(lib().znni_conv3d_fft_call_work_v, S, f, fo, n, k, _flags(relu, mac_reference, keep_kernels))


def _work(fn, S, f, fo, n, k, flags):
    nb = (ctypes.c_double * len(STAGES))()
    fl = (ctypes.c_double * len(STAGES))()
    _check(fn(int(S), int(f), int(fo), _triple(n), _triple(k), flags, nb, fl))
    return ({name: float(nb[q]) for q, name in enumerate(STAGES)},
            {name: float(fl[q]) for q, name in enumerate(STAGES)})


def znni_conv3d_fft_sublayers(S, f, fo, n, k, budget_bytes):
    """Division of a layer for a workspace budget: ((S_i, f_i, f'_i), workspace bytes needed)."""
    sub = (ctypes.c_int * 3)()
    b = ctypes.c_size_t(0)
    _check(lib().znni_conv3d_fft_sublayers_v(int(S), int(f), int(fo), _triple(n), _triple(k), int(budget_bytes),
                                             sub, ctypes.byref(b)))
    return tuple(sub), int(b.value)


def znni_conv3d_fft_budget(inp, w, bias=None, relu=False, out=None, workspace=None, stream=None,
                           mac_reference=False):
    """The layer computed as sub-layers that fit `workspace` (a torch uint8 CUDA tensor, required)."""
    assert workspace is not None, "the workspace is the budget"
    S, f, fo, n, k, out, workspace = _marshal(inp, w, bias, out, workspace)
    st = stream if stream is not None else torch.cuda.current_stream(inp.device)
    _check(lib().znni_conv3d_fft_budget_v(S, f, fo, _triple(n), _triple(k), inp.data_ptr(), w.data_ptr(),
                                          bias.data_ptr() if bias is not None else None, out.data_ptr(),
                                          _flags(relu, mac_reference), workspace.data_ptr(), workspace.numel(),
                                          st.cuda_stream))
    return out


def znni_conv3d_direct_workspace(S, f, fo, n, k):
    b = ctypes.c_size_t(0)
    _check(lib().znni_conv3d_direct_workspace_v(int(S), int(f), int(fo), _triple(n), _triple(k), ctypes.byref(b)))
    return int(b.value)


def znni_conv3d_direct(inp, w, bias=None, relu=False, out=None, workspace=None, stream=None):
    """The layer by direct convolution on the matrix cores (same tensors and result as znni_conv3d_fft)."""
    assert inp.is_cuda and inp.dtype == torch.float32 and inp.is_contiguous() and inp.dim() == 5
    S, f = inp.shape[0], inp.shape[1]
    if workspace is None:
        workspace = torch.empty(znni_conv3d_direct_workspace(S, f, w.shape[0], tuple(inp.shape[2:]), tuple(w.shape[2:])),
                                dtype=torch.uint8, device=inp.device)
    S, f, fo, n, k, out, workspace = _marshal(inp, w, bias, out, workspace)
    st = stream if stream is not None else torch.cuda.current_stream(inp.device)
    _check(lib().znni_conv3d_direct_v(S, f, fo, _triple(n), _triple(k), inp.data_ptr(), w.data_ptr(),
                                      bias.data_ptr() if bias is not None else None, out.data_ptr(),
                                      RELU if relu else 0, workspace.data_ptr(), workspace.numel(), st.cuda_stream))
    return out


PRIMITIVES = ("fft", "direct")


def znni_conv3d_choose(S, f, fo, n, k):
    """(name of the primitive picked for this layer shape, {name: estimated milliseconds})."""
    prim = ctypes.c_int(0)
    est = (ctypes.c_float * 2)()
    _check(lib().znni_conv3d_choose_v(int(S), int(f), int(fo), _triple(n), _triple(k), ctypes.byref(prim), est))
    return PRIMITIVES[prim.value], {name: float(est[q]) for q, name in enumerate(PRIMITIVES)}


def znni_conv3d(inp, w, bias=None, relu=False, out=None, stream=None):
    """The layer by whichever primitive the library picks for its shape."""
    assert inp.is_cuda and inp.dtype == torch.float32 and inp.is_contiguous() and inp.dim() == 5
    assert w.is_cuda and w.dtype == torch.float32 and w.is_contiguous() and w.dim() == 5
    S, f, fo = inp.shape[0], inp.shape[1], w.shape[0]
    n, k = tuple(inp.shape[2:]), tuple(w.shape[2:])
    b = ctypes.c_size_t(0)
    _check(lib().znni_conv3d_workspace_v(S, f, fo, _triple(n), _triple(k), ctypes.byref(b)))
    ws = torch.empty(int(b.value), dtype=torch.uint8, device=inp.device)
    S, f, fo, n, k, out, ws = _marshal(inp, w, bias, out, ws)
    st = stream if stream is not None else torch.cuda.current_stream(inp.device)
    _check(lib().znni_conv3d_v(S, f, fo, _triple(n), _triple(k), inp.data_ptr(), w.data_ptr(),
                               bias.data_ptr() if bias is not None else None, out.data_ptr(),
                               RELU if relu else 0, ws.data_ptr(), ws.numel(), st.cuda_stream))
    return out


def _pool(fn, inp, p, oshape, out, stream):
    assert inp.is_cuda and inp.dtype == torch.float32 and inp.is_contiguous() and inp.dim() == 5
    S, f = inp.shape[0], inp.shape[1]
    n = tuple(int(e) for e in inp.shape[2:])
    p = tuple(int(e) for e in _triple(p))
    shape = oshape(S, f, n, p)
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=inp.device)
    else:
        assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and tuple(out.shape) == shape
    st = stream if stream is not None else torch.cuda.current_stream(inp.device)
    _check(fn(S, f, _triple(n), _triple(p), inp.data_ptr(), out.data_ptr(), st.cuda_stream))
    return out


def znni_mpf(inp, p, out=None, stream=None):
    """Max-pooling fragments with window p (edge or (px,py,pz)): [S,f,nx,ny,nz] -> [S*px*py*pz, f, n//p ...]."""
    return _pool(lib().znni_mpf, inp, p,
                 lambda S, f, n, p: (S * p[0] * p[1] * p[2], f) + tuple(max(a // max(b, 1), 0) for a, b in zip(n, p)),
                 out, stream)


def znni_maxpool(inp, p, out=None, stream=None):
    """Max pooling with window p: [S,f,nx,ny,nz] -> [S, f, nx/px, ny/py, nz/pz]."""
    return _pool(lib().znni_maxpool, inp, p,
                 lambda S, f, n, p: (S, f) + tuple(max(a // max(b, 1), 0) for a, b in zip(n, p)), out, stream)


def znni_copy_probe(dst, src, stream=None):
    """Plain device copy src -> dst (same-size contiguous CUDA tensors); used to calibrate traffic counters."""
    assert dst.is_cuda and src.is_cuda and dst.is_contiguous() and src.is_contiguous()
    nbytes = src.numel() * src.element_size()
    assert nbytes == dst.numel() * dst.element_size()
    st = stream if stream is not None else torch.cuda.current_stream(src.device)
    _check(lib().znni_copy_probe(dst.data_ptr(), src.data_ptr(), nbytes, st.cuda_stream))
    return dst


# The attention operators.  Each call is asynchronous on `stream` (a torch.cuda.Stream of the tensors' GPU; default: torch's current
# stream).  Inputs have to be there in that stream's order; results made by the call belong to it.
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_byref = ctypes.byref
_descriptor = struct.Struct("Pqq").pack          # a znni_heads (data, token stride, head stride) as bytes


def _kind(x):
    """(znni_type, dtype, device) of a tensor of heads."""
    assert x.is_cuda and x.dtype in _TYPES, "heads are float32, bfloat16 or float16 tensors on the GPU"
    return _TYPES[x.dtype], x.dtype, x.get_device()


def _heads(x, shape, kind):
    """The znni_heads of a [tokens, heads, D] tensor of this shape and kind whose last index is contiguous."""
    assert x.shape == shape and x.dtype == kind[1] and x.get_device() == kind[2], f"need {kind[1]} heads {tuple(shape)} on GPU {kind[2]}"
    token, head, unit = x.stride()
    assert unit == 1, "tensors of heads are [tokens, heads, D], D contiguous"
    # the stride of an axis of one element (or of none) says nothing, and torch may report any
    return _descriptor(x.data_ptr(), token if shape[0] > 1 else 0, head if shape[1] > 1 else 0)


def _result(like, given, shape, kind):
    """(tensor for a result like this one of that shape and kind, its znni_heads)."""
    if given is not None:
        return given, _heads(given, shape, kind)
    out = torch.empty_like(like) if like.is_contiguous() else torch.empty_like(like, memory_format=torch.contiguous_format)
    return out, _descriptor(out.data_ptr(), shape[1] * shape[2], shape[2])


def _ints(x, kind, *shape):
    assert x.get_device() == kind[2] and x.dtype == torch.int32 and x.shape == shape and x.is_contiguous(), \
        f"need contiguous int32 {shape} on GPU {kind[2]}"
    return x.data_ptr()


def _window(v):
    return ALL if v is None else int(v)


def _current(x):
    """The stream to launch on: torch's current one."""
    return torch._C._cuda_getCurrentRawStream(x.get_device())


def _on(stream, x, call, *args, **kw):
    """`call` with `stream` as torch's current one: all that it copies and allocates is ordered with its launches.  Results belong to
    that stream then, and stay until the caller's own stream has used them."""
    assert stream.device == x.device, f"need a stream of {x.device}"
    callers = torch.cuda.current_stream(x.device)
    with torch.cuda.stream(stream):
        results = call(*args, **kw)
    for r in results if isinstance(results, tuple) else (results,):
        if r is not None:
            r.record_stream(callers)
    return results


def _scratch(need, workspace, x):
    """(address, bytes) of the caller's workspace or of one made here, and the tensor."""
    if workspace is None:
        if not need:
            return None, 0, None
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
        return workspace.data_ptr(), need, workspace
    assert workspace.get_device() == x.get_device() and workspace.dtype == torch.uint8 and workspace.is_contiguous()
    return workspace.data_ptr(), workspace.numel(), workspace


@functools.lru_cache(4096)
def _need(L, query, *args):
    """Bytes that a workspace query of the library answers for these sizes."""
    b = ctypes.c_size_t(0)
    _check(getattr(L, query)(*args, _byref(b)))
    return b.value


def znni_rope_axes(q, k, pos, freq, sections, pairing="halves", out_q=None, out_k=None, stream=None):
    """Rotary positions with several axes on q [T, Hq, D] and k [T, Hk, D] (k may be None): pair j is turned by
    pos[t, a] * freq[j], a the axis whose section holds j.  pairing: "halves" (j, R + j) or "neighbours" (2j, 2j + 1), R the sum
    of sections.  pos int32 [T, axes], signed; freq float32 [R].  out_q, out_k may be q and k.  Returns (out_q, out_k)."""
    if stream is not None:
        return _on(stream, q, znni_rope_axes, q, k, pos, freq, sections, pairing, out_q, out_k)
    kind = _kind(q)
    T, Hq, D = shape = q.shape
    axes = len(sections)
    out_q, do_q = _result(q, out_q, shape, kind)
    Hk, dk, do_k = 0, None, None
    if k is not None:
        kshape = k.shape
        Hk = kshape[1]
        assert kshape == (T, Hk, D)
        dk = _heads(k, kshape, kind)
        out_k, do_k = _result(k, out_k, kshape, kind)
    assert freq.get_device() == kind[2] and freq.dtype == torch.float32 and freq.is_contiguous() and freq.shape == (sum(sections),)
    _check(lib().znni_rope_axes(kind[0], T, Hq, Hk, D, _heads(q, shape, kind), dk, _ints(pos, kind, T, axes), freq.data_ptr(), axes,
                                struct.pack("%di" % axes, *sections), do_q, do_k, _PAIRINGS[pairing], _current(q)))
    return out_q, out_k


def _attn_window_need(type, B, Hq, Hk, D, max_q, max_k, left, right, sinks):
    b = ctypes.c_size_t(0)
    _check(lib().znni_attn_window_workspace(type, B, Hq, Hk, D, max_q, max_k, left, right, sinks, _byref(b)))
    return b.value


def znni_attn_window_workspace(dtype, B, Hq, Hk, D, max_q, max_k, left=None, right=0, sinks=0):
    return _attn_window_need(_TYPES[dtype], int(B), int(Hq), int(Hk), int(D), int(max_q), int(max_k), _window(left), _window(right), int(sinks))


def znni_attn_window(q, k, v, cu_q, cu_k, max_q, max_k, left=None, right=0, sinks=0, scale=None, out=None, workspace=None,
                     stream=None, stats=None):
    """Attention over B sequences one behind the other: q [Tq, Hq, D], k and v [Tk, Hk, D], cu_q and cu_k int32 [B + 1] their
    starts.  The last query of a sequence stands at its last key; a row at position p sees keys p - left .. p + right (None:
    without an end) and, up to p + right, the first `sinks` keys.  Rows that see nothing are zero.  scale: D ** -0.5.
    stats: True returns (out, stats), float32 [Tq, Hq, 2], which the gradients need (or the tensor to put them in)."""
    if stream is not None:
        return _on(stream, q, znni_attn_window, q, k, v, cu_q, cu_k, max_q, max_k, left, right, sinks, scale, out, workspace, None, stats)
    Tq, Hq, D = q.shape
    Tk, Hk, _ = k.shape
    B = cu_q.numel() - 1
    assert k.shape == v.shape and k.shape[2] == D
    left, right, sinks = _window(left), _window(right), int(sinks)
    max_q, max_k = int(max_q) if Tq else 0, int(max_k) if Tk else 0          # tensors of no tokens have no address
    kind = _kind(q)
    out, do = _result(q, out, q.shape, kind)
    w, n, held = _scratch(_attn_window_need(kind[0], B, Hq, Hk, D, max_q, max_k, left, right, sinks), workspace, q)
    args = (kind[0], B, Hq, Hk, D, _heads(q, q.shape, kind), _heads(k, k.shape, kind), _heads(v, k.shape, kind), _ints(cu_q, kind, B + 1),
            _ints(cu_k, kind, B + 1), max_q, max_k, left, right, sinks, D ** -0.5 if scale is None else scale, do)
    if stats is None:
        _check(lib().znni_attn_window(*args, w, n, _current(q)))
        return out
    stats = torch.empty((Tq, Hq, 2), dtype=torch.float32, device=q.device) if stats is True else stats
    _check(lib().znni_attn_window_stats(*args, _stats(stats, Tq, Hq, kind), w, n, _current(q)))
    return out, stats


def _stats(stats, Tq, Hq, kind):
    assert stats.shape == (Tq, Hq, 2) and stats.dtype == torch.float32 and stats.get_device() == kind[2] and stats.is_contiguous(), \
        f"need contiguous float32 statistics {(Tq, Hq, 2)} on GPU {kind[2]}"
    return stats.data_ptr()


def znni_attn_window_backward_workspace(dtype, B, Hq, Hk, D, max_q, max_k, left=None, right=0, sinks=0):
    return _need(lib(), "znni_attn_window_backward_workspace", _TYPES[dtype], int(B), int(Hq), int(Hk), int(D), int(max_q), int(max_k), _window(left), _window(right), int(sinks))


def znni_attn_window_backward(dout, q, k, v, out, stats, cu_q, cu_k, max_q, max_k, left=None, right=0, sinks=0, scale=None, dq=None, dk=None,
                              dv=None, workspace=None, stream=None):
    """Gradients (dq, dk, dv) of znni_attn_window from its result's, dout; out and stats are what that call gave (stats=True), all else as it had it."""
    if stream is not None:
        return _on(stream, q, znni_attn_window_backward, dout, q, k, v, out, stats, cu_q, cu_k, max_q, max_k, left, right, sinks, scale, dq, dk, dv,
                   workspace)
    Tq, Hq, D = shape = q.shape
    Tk, Hk, _ = kshape = k.shape
    B = cu_q.numel() - 1
    assert v.shape == kshape and kshape[2] == D
    left, right, sinks = _window(left), _window(right), int(sinks)
    max_q, max_k = int(max_q) if Tq else 0, int(max_k) if Tk else 0          # tensors of no tokens have no address
    kind = _kind(q)
    dq, do_q = _result(q, dq, shape, kind)
    dk, do_k = _result(k, dk, kshape, kind)
    dv, do_v = _result(v, dv, kshape, kind)
    w, n, held = _scratch(_need(lib(), "znni_attn_window_backward_workspace", kind[0], B, Hq, Hk, D, max_q, max_k, left, right, sinks), workspace, q)
    _check(lib().znni_attn_window_backward(kind[0], B, Hq, Hk, D, _heads(q, shape, kind), _heads(k, kshape, kind), _heads(v, kshape, kind),
                                           _heads(out, shape, kind), _stats(stats, Tq, Hq, kind), _heads(dout, shape, kind), _ints(cu_q, kind, B + 1),
                                           _ints(cu_k, kind, B + 1), max_q, max_k, left, right, sinks, D ** -0.5 if scale is None else scale,
                                           do_q, do_k, do_v, w, n, _current(q)))
    return dq, dk, dv


def kv8_alloc(pages, Hk, D, device="cuda"):
    """(kcodes, vcodes, scales) of an 8-bit cache: codes [pages, Hk, 64, D] for keys, [pages, Hk, D, 64] for values, scales
    [pages, Hk, 2] for keys and values.  Contents are whatever the memory holds: appending tokens defines them."""
    return (torch.empty((pages, Hk, KV8_PAGE, D), dtype=torch.uint8, device=device),
            torch.empty((pages, Hk, D, KV8_PAGE), dtype=torch.uint8, device=device),
            torch.empty((pages, Hk, 2), dtype=torch.float32, device=device))


def _cache(kcodes, vcodes, scales, Hk, D, kind):
    """Addresses of a cache's three tensors, and its pages."""
    pages = kcodes.shape[0]
    assert kcodes.dtype == vcodes.dtype == torch.uint8 and scales.dtype == torch.float32
    assert kcodes.is_contiguous() and vcodes.is_contiguous() and scales.is_contiguous()
    assert kcodes.get_device() == vcodes.get_device() == scales.get_device() == kind[2], f"need a cache on GPU {kind[2]}"
    assert kcodes.shape == (pages, Hk, KV8_PAGE, D) and vcodes.shape == (pages, Hk, D, KV8_PAGE) and scales.shape == (pages, Hk, 2)
    return kcodes.data_ptr(), vcodes.data_ptr(), scales.data_ptr(), pages


def znni_kv8_append(kcodes, vcodes, scales, k, v, table, cu, start, max_new, stream=None):
    """Puts k, v [T, Hk, D] (cu int32 [B + 1]: where each sequence's tokens start) into the cache behind the start[b] tokens
    that sequence b holds; table int32 [B, width] names its pages.  max_new: no sequence gets more."""
    if stream is not None:
        return _on(stream, k, znni_kv8_append, kcodes, vcodes, scales, k, v, table, cu, start, max_new)
    T, Hk, D = k.shape
    B, width = table.shape
    kind = _kind(k)
    kc, vc, sc, pages = _cache(kcodes, vcodes, scales, Hk, D, kind)
    _check(lib().znni_kv8_append(kind[0], B, Hk, D, _heads(k, k.shape, kind), _heads(v, k.shape, kind), _ints(cu, kind, B + 1), _ints(start, kind, B),
                                 int(max_new) if T else 0, kc, vc, sc, pages, _ints(table, kind, B, width), width, _current(k)))


def _kv8_attn_need(type, B, Lq, Hq, Hk, D, max_len, left, sinks):
    b = ctypes.c_size_t(0)
    _check(lib().znni_kv8_attn_workspace(type, B, Lq, Hq, Hk, D, max_len, left, sinks, _byref(b)))
    return b.value


def znni_kv8_attn_workspace(dtype, B, Lq, Hq, Hk, D, max_len, left=None, sinks=0):
    return _kv8_attn_need(_TYPES[dtype], int(B), int(Lq), int(Hq), int(Hk), int(D), int(max_len), _window(left), int(sinks))


def znni_kv8_attn(q, kcodes, vcodes, scales, table, lens, max_len, left=None, sinks=0, scale=None, out=None, workspace=None,
                  stream=None):
    """Attention of the last Lq tokens of each of B sequences, q [B, Lq, Hq, D], over the 8-bit cache.  lens int32 [B]: tokens
    of each sequence, the last Lq among them; max_len: no sequence is longer.  Visibility as for znni_attn_window, right = 0."""
    if stream is not None:
        return _on(stream, q, znni_kv8_attn, q, kcodes, vcodes, scales, table, lens, max_len, left, sinks, scale, out, workspace)
    B, Lq, Hq, D = q.shape
    Hk, width = kcodes.shape[1], table.shape[1]
    kind = _kind(q)
    kc, vc, sc, pages = _cache(kcodes, vcodes, scales, Hk, D, kind)
    left, sinks, max_len = _window(left), int(sinks), int(max_len)
    shape, rows = (B * Lq, Hq, D), q
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    assert out.shape == q.shape and out.dtype == q.dtype and out.get_device() == kind[2] and out.is_contiguous()
    token, head, unit = q.stride()[1:]
    if unit != 1 or (B > 1 and Lq > 1 and q.stride(0) != Lq * token):
        rows = q.contiguous()                        # tokens that are not evenly spaced
        token, head = Hq * D, D
    elif Lq == 1:
        token = q.stride(0)
    dq = _descriptor(rows.data_ptr(), token if shape[0] > 1 else 0, head if Hq > 1 else 0)
    w, n, held = _scratch(_kv8_attn_need(kind[0], B, Lq, Hq, Hk, D, max_len, left, sinks), workspace, q)
    _check(lib().znni_kv8_attn(kind[0], B, Lq, Hq, Hk, D, dq, kc, vc, sc, pages, _ints(table, kind, B, width), width, _ints(lens, kind, B), max_len, left,
                               sinks, D ** -0.5 if scale is None else scale, _descriptor(out.data_ptr(), Hq * D, D), w, n,
                               _current(q)))
    return out


# Products with weights and norms between blocks: what is said of streams at the attention operators holds.
_rows_descriptor = struct.Struct("Pq").pack      # a znni_rows (data, row stride) as bytes


def _rows(x, shape, kind):
    """The znni_rows of a [rows, columns] tensor of this shape and kind whose last index is contiguous; None for None."""
    if x is None:
        return None
    assert x.shape == shape and x.dtype == kind[1] and x.get_device() == kind[2], f"need {kind[1]} rows {tuple(shape)} on GPU {kind[2]}"
    rows, cols = shape
    if x.is_contiguous():
        return _rows_descriptor(x.data_ptr(), cols)
    row, unit = x.stride()
    assert unit == 1 or cols < 2, "matrices are [rows, columns], columns contiguous"
    return _rows_descriptor(x.data_ptr(), row if rows > 1 else cols)


def _vector(x, n, kind):
    """The address of a contiguous vector; None for None."""
    if x is None:
        return None
    assert x.shape == (n,) and x.dtype == kind[1] and x.get_device() == kind[2] and x.is_contiguous(), f"need a contiguous {kind[1]} vector of {n} on GPU {kind[2]}"
    return x.data_ptr()


def znni_linear_workspace(dtype, M, N, K):
    return _need(lib(), "znni_linear_workspace", _TYPES[dtype], int(M), int(N), int(K))


def znni_linear(x, w, bias=None, act=None, residual=None, keep=False, out=None, workspace=None, stream=None):
    """residual + act(x w^T + bias): x [M, K], w [N, K], bias [N], residual [M, N] (may be `out`); act: None, "relu", "gelu" (by erf) or
    "silu".  keep: returns (out, z) with z = x w^T + bias, which the gradients need (or the tensor to put it in)."""
    if stream is not None:
        return _on(stream, x, znni_linear, x, w, bias, act, residual, keep, out, workspace)
    kind = _kind(x)
    M, K = xs = x.shape
    N = w.shape[0]
    shape = (M, N)
    out = x.new_empty(M, N) if out is None else out
    z = None if keep is False else x.new_empty(M, N) if keep is True else keep
    p, n, held = _scratch(_need(lib(), "znni_linear_workspace", kind[0], M, N, K), workspace, x)
    _check(lib().znni_linear(kind[0], M, N, K, _rows(x, xs, kind), _rows(w, (N, K), kind), _vector(bias, N, kind), _ACTIVATIONS[act],
                             _rows(residual, shape, kind), _rows(z, shape, kind), _rows(out, shape, kind), p, n, _current(x)))
    return out if z is None else (out, z)


def znni_linear_backward_workspace(dtype, M, N, K, act=None, wanted=LINEAR_DX | LINEAR_DW | LINEAR_DBIAS):
    return _need(lib(), "znni_linear_backward_workspace", _TYPES[dtype], int(M), int(N), int(K), _ACTIVATIONS[act], int(wanted))


def znni_linear_backward(dout, x, w, z=None, act=None, bias=True, inputs=True, weights=True, dx=None, dw=None, dbias=None, workspace=None,
                         stream=None):
    """Gradients (dx, dw, dbias) of znni_linear from its result's, dout [M, N]; None for those that `inputs`, `weights` and `bias` do not ask
    for; x and w may be None where only others need them.  z: what the forward call kept (with an activation).  The residual's gradient is dout."""
    if stream is not None:
        return _on(stream, dout, znni_linear_backward, dout, x, w, z, act, bias, inputs, weights, dx, dw, dbias, workspace)
    kind = _kind(dout)
    M, N = shape = dout.shape
    K = w.shape[1] if w is not None else x.shape[1] if x is not None else 0          # (the bias's gradient takes neither)
    dx = (dout.new_empty(M, K) if dx is None else dx) if inputs else None
    dw = (dout.new_empty(N, K) if dw is None else dw) if weights else None
    dbias = (dout.new_empty(N) if dbias is None else dbias) if bias else None
    wanted = (LINEAR_DX if inputs else 0) | (LINEAR_DW if weights else 0) | (LINEAR_DBIAS if bias else 0)
    a = _ACTIVATIONS[act]
    p, n, held = _scratch(_need(lib(), "znni_linear_backward_workspace", kind[0], M, N, K, a, wanted), workspace, dout)
    _check(lib().znni_linear_backward(kind[0], M, N, K, _rows(dout, shape, kind), _rows(x, (M, K), kind), _rows(w, (N, K), kind),
                                      _rows(z, shape, kind), a, _rows(dx, (M, K), kind), _rows(dw, (N, K), kind), _vector(dbias, N, kind), p, n,
                                      _current(dout)))
    return dx, dw, dbias


def _gate(gate, shape, kind):
    """(whether one gate is for all tokens, its znni_rows)."""
    if gate is None:
        return 0, None
    if gate.dim() == 1:
        return NORM_GATE_SHARED, _rows_descriptor(_vector(gate, shape[1], kind), shape[1])
    return 0, _rows(gate, shape, kind)


def znni_block_norm(x, y=None, gate=None, post=None, pre=None, scale=1.0, eps=1e-5, centred=False, norm_post=True, norm_pre=True, h=None,
                    z=None, stream=None):
    """(h, z): h = x + scale * gate * post * n(y), z = pre * n(h), for x, y [T, C], gate [T, C] or [C], post and pre [C] (None: ones).
    n divides a row by its root mean square, or, `centred`, takes its mean off and divides it by its deviation.  Without norm_post y is taken as
    it is, without norm_pre there is no z (None).  y None: there is no block, and h is x."""
    if stream is not None:
        return _on(stream, x, znni_block_norm, x, y, gate, post, pre, scale, eps, centred, norm_post, norm_pre, h, z)
    kind = _kind(x)
    T, C = shape = x.shape
    shared, dg = _gate(gate, shape, kind)
    norm_post = norm_post and y is not None
    flags = (NORM_POST if norm_post else 0) | (NORM_PRE if norm_pre else 0) | (NORM_CENTRED if centred else 0) | shared
    h = x if y is None else x.new_empty(T, C) if h is None else h
    z = (x.new_empty(T, C) if z is None else z) if norm_pre else None
    _check(lib().znni_block_norm(kind[0], T, C, _rows(x, shape, kind), _rows(y, shape, kind), dg, _vector(post, C, kind), _vector(pre, C, kind), scale, eps,
                                 flags, _rows(h, shape, kind) if y is not None else None, _rows(z, shape, kind), _current(x)))
    return h, z


def znni_block_norm_backward_workspace(dtype, T, C):
    return _need(lib(), "znni_block_norm_backward_workspace", _TYPES[dtype], int(T), int(C), 0)


def znni_block_norm_backward(dh, dz, h, y=None, gate=None, post=None, pre=None, scale=1.0, eps=1e-5, centred=False, norm_post=True,
                             norm_pre=True, dx=None, dy=None, dgate=None, dpost=None, dpre=None, workspace=None, stream=None):
    """Gradients (dx, dy, dgate, dpost, dpre) of znni_block_norm from those of its results, dh (None: zero) and dz, and from h and y as it had
    them; None for what the call does not have."""
    if stream is not None:
        return _on(stream, h, znni_block_norm_backward, dh, dz, h, y, gate, post, pre, scale, eps, centred, norm_post, norm_pre, dx, dy, dgate, dpost, dpre, workspace)
    kind = _kind(h)
    T, C = shape = h.shape
    shared, dg = _gate(gate, shape, kind)
    norm_post = norm_post and y is not None
    flags = (NORM_POST if norm_post else 0) | (NORM_PRE if norm_pre else 0) | (NORM_CENTRED if centred else 0) | shared
    dx = h.new_empty(T, C) if dx is None else dx
    dy = (h.new_empty(T, C) if dy is None else dy) if y is not None else None
    dgate = (h.new_empty(gate.shape) if dgate is None else dgate) if gate is not None else None
    dpost = (h.new_empty(C) if dpost is None else dpost) if post is not None else None
    dpre = (h.new_empty(C) if dpre is None else dpre) if pre is not None else None
    summed = shared or dpost is not None or dpre is not None
    p, n, held = _scratch(_need(lib(), "znni_block_norm_backward_workspace", kind[0], T, C, flags) if summed else 0, workspace, h)
    _check(lib().znni_block_norm_backward(kind[0], T, C, _rows(dh, shape, kind), _rows(dz, shape, kind), _rows(h, shape, kind), _rows(y, shape, kind), dg,
                                          _vector(post, C, kind), _vector(pre, C, kind), scale, eps, flags, _rows(dx, shape, kind),
                                          _rows(dy, shape, kind), _gate(dgate, shape, kind)[1], _vector(dpost, C, kind), _vector(dpre, C, kind), p, n,
                                          _current(h)))
    return dx, dy, dgate, dpost, dpre
