"""ctypes binding of liboaa.so (include/oaa.h). Argument marshalling only.

Functions carry the C names and take plain integers for device pointers and
streams. ``Plan``, ``group_norm_*`` and ``grad_*`` wrap them for torch tensors:
torch supplies device memory (workspaces are uint8 tensors) and the current
stream; every step of every pass runs in the library's HIP kernels. There is no fallback: if the library
is missing, ``load()`` raises.
"""

import array
import ctypes
import functools
import math
import os

from .build import LIB_PATH

OAA_OK = 0
STATUS = {0: "OAA_OK", 1: "OAA_ERR_INVALID_ARG", 2: "OAA_ERR_UNSUPPORTED",
          3: "OAA_ERR_NO_WORKSPACE", 4: "OAA_ERR_NO_CACHE", 5: "OAA_ERR_HIP"}
REGION_W_SPECTRUM, REGION_X_SPECTRUM, REGION_G_SPECTRUM, REGION_PRODUCT = 0, 1, 2, 3
CONTRACTION_AUTO, CONTRACTION_VALU, CONTRACTION_MFMA, CONTRACTION_NARROW, CONTRACTION_FUSED = 0, 1, 2, 3, 4
METHOD_OVERLAP_ADD, METHOD_OVERLAP_SAVE = 0, 1
STAGES = ["w_spectrum", "x_spectrum", "g_spectrum", "fwd_product", "fwd_inverse",
          "bwd_data_product", "bwd_data_inverse", "bwd_filter_product", "bwd_filter_inverse"]

LAYOUT_PLANES, LAYOUT_CHANNELS_LAST = 0, 1
FLOAT32, BFLOAT16, FLOAT16 = 0, 1, 2
ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
NORM_SUM, NORM_EUCLIDEAN, NORM_MAX = 1, 2, 3

# every symbol include/oaa.h declares, with its ctypes signature
_c_int, _c_size, _vp = ctypes.c_int, ctypes.c_size_t, ctypes.c_void_p


class Geometry(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int) for k in ("B", "C", "K", "N", "n", "M", "T", "P", "L", "F", "split", "b",
                                            "method", "fused")]


class Strides(ctypes.Structure):
    _fields_ = [("image", ctypes.c_longlong), ("row", ctypes.c_longlong)]


class GroupNormDesc(ctypes.Structure):
    """oaa_group_norm_t."""
    _fields_ = [("B", ctypes.c_int), ("C", ctypes.c_int), ("G", ctypes.c_int), ("S", ctypes.c_longlong),
                ("layout", ctypes.c_int), ("dtype", ctypes.c_int), ("param_dtype", ctypes.c_int),
                ("activation", ctypes.c_int), ("eps", ctypes.c_float),
                ("x", Strides), ("y", Strides), ("dy", Strides), ("dx", Strides)]


SIGNATURES = {
    "oaa_plan_create": (_c_int, [ctypes.POINTER(_vp), _c_int, _c_int, _c_int, _c_int, _c_int]),
    "oaa_plan_create_tiled": (_c_int, [ctypes.POINTER(_vp), _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int]),
    "oaa_plan_create_method": (_c_int, [ctypes.POINTER(_vp), _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int,
                                        _c_int]),
    "oaa_plan_destroy": (_c_int, [_vp]),
    "oaa_plan_geometry": (_c_int, [_vp, ctypes.POINTER(Geometry)]),
    "oaa_plan_workspace_bytes": (_c_size, [_vp]),
    "oaa_plan_region": (_c_int, [_vp, _c_int, ctypes.POINTER(_c_size), ctypes.POINTER(_c_size)]),
    "oaa_plan_bind_workspace": (_c_int, [_vp, _vp, _c_size]),
    "oaa_plan_set_contraction": (_c_int, [_vp, _c_int]),
    "oaa_plan_set_timing": (_c_int, [_vp, _c_int]),
    "oaa_plan_stage_times": (_c_int, [_vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(_c_int), _c_int]),
    "oaa_conv_forward": (_c_int, [_vp, _vp, _vp, _vp, _vp]),
    "oaa_conv_backward_data": (_c_int, [_vp, _vp, _vp, _vp, _vp]),
    "oaa_conv_backward_filter": (_c_int, [_vp, _vp, _vp, _vp, _vp]),
    "oaa_conv_forward_noalloc": (_c_int, [_vp, _vp, _vp, _vp, _vp]),
    "oaa_plan_chain_scratch_bytes": (_c_size, [_vp, _c_int]),
    "oaa_plan_set_kernel_chain": (_c_int, [_vp, _vp, _c_int, _c_int, _vp, _c_int, _vp, _c_size, _vp]),
    "oaa_group_norm_workspace_bytes": (_c_size, [_vp, _c_int]),
    "oaa_group_norm_forward": (_c_int, [_vp] * 8 + [_c_size, _vp]),
    "oaa_group_norm_backward": (_c_int, [_vp] * 11 + [_c_size, _vp]),
    "oaa_grad_workspace_bytes": (_c_size, [_c_int]),
    "oaa_grad_norm": (_c_int, [_c_int, _vp, _vp, _vp, _c_int, _vp, _vp, _c_size, _vp]),
    "oaa_grad_clip": (_c_int, [_c_int, _vp, _vp, _vp, _vp, _c_int, ctypes.c_float, _vp, _vp, _c_size, _vp]),
    "oaa_status_string": (ctypes.c_char_p, [_c_int]),
    "oaa_last_error_detail": (ctypes.c_char_p, []),
}

_LIB = None


def load(path=None):
    """Load liboaa.so (once) and declare its signatures."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    path = path or LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run paper_1601_06815_amd.build.build() "
                           "(or __graft_entry__.build()) first")
    lib = ctypes.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if path == LIB_PATH:
        _LIB = lib
    return lib


def use_library(path):
    """Load liboaa.so from `path` and make it the library every later call
    uses (for comparing builds; the default is the in-tree build)."""
    global _LIB
    _LIB = None
    lib = load(path)
    _LIB = lib
    return lib


class OaaError(RuntimeError):
    def __init__(self, status, detail):
        super().__init__(f"{STATUS.get(status, status)}: {detail}")
        self.status = status
        self.detail = detail


def _check(st):
    if st != OAA_OK:
        lib = load()
        raise OaaError(st, lib.oaa_last_error_detail().decode())
    return st


# ---- C names, integer pointers ------------------------------------------------

def oaa_plan_create(B, C, K, N, n):
    h = _vp()
    _check(load().oaa_plan_create(ctypes.byref(h), B, C, K, N, n))
    return h.value


def oaa_plan_create_tiled(B, C, K, N, n, L, b):
    h = _vp()
    _check(load().oaa_plan_create_tiled(ctypes.byref(h), B, C, K, N, n, L, b))
    return h.value


def oaa_plan_create_method(B, C, K, N, n, L, b, method):
    h = _vp()
    _check(load().oaa_plan_create_method(ctypes.byref(h), B, C, K, N, n, L, b, method))
    return h.value


def oaa_plan_destroy(plan):
    return _check(load().oaa_plan_destroy(plan))


def oaa_plan_geometry(plan):
    g = Geometry()
    _check(load().oaa_plan_geometry(plan, ctypes.byref(g)))
    return {k: getattr(g, k) for k, _ in Geometry._fields_}


def oaa_plan_workspace_bytes(plan):
    return load().oaa_plan_workspace_bytes(plan)


def oaa_plan_region(plan, region):
    off, size = _c_size(), _c_size()
    _check(load().oaa_plan_region(plan, region, ctypes.byref(off), ctypes.byref(size)))
    return off.value, size.value


def oaa_plan_bind_workspace(plan, dev_ptr, nbytes):
    return _check(load().oaa_plan_bind_workspace(plan, dev_ptr, nbytes))


def oaa_plan_set_contraction(plan, which):
    return _check(load().oaa_plan_set_contraction(plan, which))


def oaa_plan_set_timing(plan, enable):
    return _check(load().oaa_plan_set_timing(plan, 1 if enable else 0))


def oaa_plan_stage_times(plan):
    """{stage name: (total ms, launches)} since the last call; waits for the GPU."""
    n = len(STAGES)
    ms = (ctypes.c_double * n)()
    cnt = (_c_int * n)()
    _check(load().oaa_plan_stage_times(plan, ms, cnt, n))
    return {name: (ms[i], cnt[i]) for i, name in enumerate(STAGES)}


def oaa_conv_forward(plan, x, w, y, stream):
    return _check(load().oaa_conv_forward(plan, x, w, y, stream))


def oaa_conv_backward_data(plan, g, w, dx, stream):
    return _check(load().oaa_conv_backward_data(plan, g, w, dx, stream))


def oaa_conv_backward_filter(plan, x, g, dw, stream):
    return _check(load().oaa_conv_backward_filter(plan, x, g, dw, stream))


def oaa_conv_forward_noalloc(plan, x, w, y, stream):
    return _check(load().oaa_conv_forward_noalloc(plan, x, w, y, stream))


def oaa_plan_chain_scratch_bytes(plan, J):
    return load().oaa_plan_chain_scratch_bytes(plan, J)


def oaa_plan_set_kernel_chain(plan, w1, J, n1, w2, n2, scratch, scratch_bytes, stream):
    return _check(load().oaa_plan_set_kernel_chain(plan, w1, J, n1, w2, n2, scratch, scratch_bytes, stream))


def oaa_group_norm_workspace_bytes(desc, backward):
    """desc: a GroupNormDesc or its address."""
    return load().oaa_group_norm_workspace_bytes(_address(desc), 1 if backward else 0)


def oaa_group_norm_forward(desc, x, weight, bias, y, mean, rstd, workspace, workspace_bytes, stream):
    return _check(load().oaa_group_norm_forward(_address(desc), x, weight, bias, y, mean, rstd, workspace,
                                                workspace_bytes, stream))


def oaa_group_norm_backward(desc, dy, x, weight, bias, mean, rstd, dx, dweight, dbias, workspace, workspace_bytes,
                            stream):
    return _check(load().oaa_group_norm_backward(_address(desc), dy, x, weight, bias, mean, rstd, dx, dweight, dbias,
                                                 workspace, workspace_bytes, stream))


def oaa_grad_workspace_bytes(count):
    return load().oaa_grad_workspace_bytes(count)


def oaa_grad_norm(count, grads, sizes, dtypes, norm_type, norm, workspace, workspace_bytes, stream):
    """grads, sizes, dtypes: addresses of host arrays."""
    return _check(load().oaa_grad_norm(count, grads, sizes, dtypes, norm_type, norm, workspace, workspace_bytes,
                                       stream))


def oaa_grad_clip(count, grads, out, sizes, dtypes, norm_type, max_norm, norm, workspace, workspace_bytes, stream):
    return _check(load().oaa_grad_clip(count, grads, out, sizes, dtypes, norm_type, max_norm, norm, workspace,
                                       workspace_bytes, stream))


def _address(desc):
    return desc if isinstance(desc, int) or desc is None else ctypes.addressof(desc)


def oaa_status_string(status):
    return load().oaa_status_string(status).decode()


def oaa_last_error_detail():
    return load().oaa_last_error_detail().decode()


# ---- torch convenience wrapper ----------------------------------------------

class Plan:
    """One layer x[B,C,N,N] (*) w[K,C,n,n]; owns a plan handle and a device
    workspace tensor. Calls enqueue on torch's current stream of the tensors'
    device and return without synchronising. The workspace is marked as used
    by every stream a call runs on, so that torch does not hand its memory
    out again before that work is done once the plan is released.
    ``generation`` counts the passes that replaced cached spectra (forward,
    backward_data, backward_filter)."""

    def __init__(self, B, C, K, N, n, device="cuda", contraction=CONTRACTION_AUTO, tiling="paper",
                 method=METHOD_OVERLAP_ADD):
        """tiling: "paper" (blocks of n, oaa_plan_create), "auto" (the
        library's choice) or an (L, b) pair (oaa_plan_create_tiled).
        method=METHOD_OVERLAP_SAVE: the output-tiled passes
        (oaa_plan_create_method); tiling "auto"/"paper" or (L, b) with b 0 or
        L - n + 1."""
        import torch
        if method != METHOD_OVERLAP_ADD:
            L, b = (0, 0) if tiling in ("paper", "auto") else tiling
            self.handle = oaa_plan_create_method(B, C, K, N, n, L, b, method)
        elif tiling == "paper":
            self.handle = oaa_plan_create(B, C, K, N, n)
        elif tiling == "auto":
            self.handle = oaa_plan_create_tiled(B, C, K, N, n, 0, 0)
        else:
            L, b = tiling
            self.handle = oaa_plan_create_tiled(B, C, K, N, n, L, b)
        self.geometry = oaa_plan_geometry(self.handle)
        self.device = torch.device(device)
        self.generation = 0
        self._torch = torch
        # shapes of the passes' tensors
        g = self.geometry
        self._x = torch.Size((g["B"], g["C"], g["N"], g["N"]))
        self._w = torch.Size((g["K"], g["C"], g["n"], g["n"]))
        self._y = torch.Size((g["B"], g["K"], g["M"], g["M"]))
        nbytes = oaa_plan_workspace_bytes(self.handle)
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        self._streams = {torch.cuda.current_stream(self.device).cuda_stream}
        oaa_plan_bind_workspace(self.handle, self.workspace.data_ptr(), self.workspace.numel())
        if contraction != CONTRACTION_AUTO:
            oaa_plan_set_contraction(self.handle, contraction)
            self.geometry = oaa_plan_geometry(self.handle)

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            try:
                oaa_plan_destroy(h)
            except Exception:
                pass
            self.handle = None

    @property
    def output_side(self):
        return self.geometry["M"]

    @property
    def caches_grad_spectra(self):
        """Whether backward_filter may take gr=None after backward_data (the
        fused few-channel passes keep no gradient spectra)."""
        return not self.geometry["fused"]

    def _ptr(self, t, shape, name):
        if t is None:
            return None
        if t.dtype != self._torch.float32 or not t.is_contiguous() or t.device != self.device:
            raise ValueError(f"{name} must be a contiguous float32 tensor on {self.device}")
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        return t.data_ptr()

    def _stream(self):
        # the raw handle: a Stream object costs several times as much, most of
        # all in autograd's backward thread
        index = self.device.index
        raw = self._torch._C._cuda_getCurrentRawStream(
            self._torch.cuda.current_device() if index is None else index)
        if raw not in self._streams:
            s = self._torch.cuda.current_stream(self.device)
            self.workspace.record_stream(s)
            self._streams.add(raw)
        return raw

    def _empty(self, shape):
        return self._torch.empty(shape, dtype=self._torch.float32, device=self.device)

    def forward(self, x, w, y=None):
        y = self._empty(self._y) if y is None else y
        oaa_conv_forward(self.handle, self._ptr(x, self._x, "x"), self._ptr(w, self._w, "w"),
                         self._ptr(y, self._y, "y"), self._stream())
        self.generation += 1
        return y

    def forward_noalloc(self, x, w, y):
        """oaa_conv_forward_noalloc into the caller's y: the library's static
        scratch instead of this plan's workspace, no allocation."""
        oaa_conv_forward_noalloc(self.handle, self._ptr(x, self._x, "x"), self._ptr(w, self._w, "w"),
                                 self._ptr(y, self._y, "y"), self._stream())
        return y

    def backward_data(self, gr, w, dx=None):
        dx = self._empty(self._x) if dx is None else dx
        oaa_conv_backward_data(self.handle, self._ptr(gr, self._y, "g"), self._ptr(w, self._w, "w"),
                               self._ptr(dx, self._x, "dx"), self._stream())
        self.generation += 1
        return dx

    def backward_filter(self, x, gr, dw=None):
        dw = self._empty(self._w) if dw is None else dw
        oaa_conv_backward_filter(self.handle, self._ptr(x, self._x, "x"), self._ptr(gr, self._y, "g"),
                                 self._ptr(dw, self._w, "dw"), self._stream())
        self.generation += 1
        return dw

    def set_kernel_chain(self, w1, w2):
        """oaa_plan_set_kernel_chain: the plan's kernel spectra become those
        of two stacked layers, w1[J,C,n1,n1] then w2[K,J,n2,n2] with
        n1 + n2 - 1 = n; forward(x, None) then computes both layers."""
        import torch
        g = self.geometry
        J, n1, n2 = w1.shape[0], w1.shape[-1], w2.shape[-1]
        p1 = self._ptr(w1, (J, g["C"], n1, n1), "w1")
        p2 = self._ptr(w2, (g["K"], J, n2, n2), "w2")
        nbytes = oaa_plan_chain_scratch_bytes(self.handle, J)
        scratch = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=self.device)
        stream = self._stream()
        # scratch is allocated on, and used on, the current stream: torch
        # reuses its memory only for work ordered after these kernels
        oaa_plan_set_kernel_chain(self.handle, p1, J, n1, p2, n2, scratch.data_ptr(), scratch.numel(), stream)
        self.generation += 1

    def set_timing(self, enable):
        oaa_plan_set_timing(self.handle, enable)

    def stage_times(self):
        return oaa_plan_stage_times(self.handle)

    def region(self, which):
        """A view of one workspace region as complex64 (for stage checks)."""
        import torch
        off, size = oaa_plan_region(self.handle, which)
        return self.workspace[off:off + size].view(torch.complex64)


# ---- group normalisation and gradients of torch tensors ------------------------

@functools.lru_cache(maxsize=None)
def _dtype_codes():
    import torch
    return {torch.float32: FLOAT32, torch.bfloat16: BFLOAT16, torch.float16: FLOAT16}


@functools.lru_cache(maxsize=None)
def _torch():
    """torch, and its calls for the current device and its raw stream."""
    import torch
    return torch, torch.cuda.current_device, torch._C._cuda_getCurrentRawStream


@functools.lru_cache(maxsize=None)
def _written():
    """torch's call that tells autograd of tensors, which a graph may have saved,
    that they changed."""
    import torch
    return torch.autograd.graph.increment_version


def _launch(fn, index, *args):
    """fn(*args, stream) on the current stream of device `index`, with that
    device current: kernels are launched there."""
    torch, current_device, raw_stream = _torch()
    if current_device() == index:
        status = fn(*args, raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, raw_stream(index))
    if status != OAA_OK:
        _check(status)


def _is_dense(shape, strides):
    expect = 1
    for k, st in zip(reversed(shape), reversed(strides)):
        if k != 1:
            if st != expect:
                return math.prod(shape) == 0
            expect *= k
    return True


def _layout_of(shape, strides, name, want=None):
    """(layout, S, image stride, row stride) of a tensor [B, C, ...], in planes or
    channels last with any strides between positions and images; `want`: only
    this layout will do (one position or one channel is both). One vector over all
    images and positions is refused: the description's strides 0 and 0 mean dense."""
    if len(shape) < 2:
        raise ValueError(f"{name} must have shape [B, C, ...], got {tuple(shape)}")
    C = shape[1]
    S = math.prod(shape[2:])
    if want != LAYOUT_CHANNELS_LAST and _is_dense(shape, strides):
        return LAYOUT_PLANES, S, C * S, S
    # the positions' dimensions as one: row-major with one step between neighbours
    step = expect = None
    for k, st in zip(reversed(shape[2:]), reversed(strides[2:])):
        if k == 1:
            continue
        if step is None:
            step = expect = st
        if st != expect:
            raise ValueError(f"{name}: positions of {tuple(shape)} with strides {strides} are not evenly spaced")
        expect *= k
    image = strides[0] if shape[0] > 1 else C * S
    if want != LAYOUT_CHANNELS_LAST and step in (None, 1) and (C == 1 or strides[1] == S):
        return LAYOUT_PLANES, S, image, S
    if want != LAYOUT_PLANES and (C == 1 or strides[1] == 1):
        row = C if step is None else step
        if image == 0 and row == 0 and S:
            raise ValueError(f"{name}: strides {strides} of {tuple(shape)} repeat one position of one image everywhere")
        return LAYOUT_CHANNELS_LAST, S, image, row
    kind = {None: "planes or channels last", LAYOUT_PLANES: "planes", LAYOUT_CHANNELS_LAST: "channels last"}[want]
    raise ValueError(f"{name}: strides {strides} of {tuple(shape)} are not {kind}")


def _norm_layout(t, name, want=None):
    return _layout_of(t.shape, t.stride(), name, want)


class _NormCall:
    """What a call works out from shapes, strides and types alone: the checks of
    them, the description and the workspaces' sizes."""

    def __init__(self, shape, strides, y_strides, dy_strides, dtype, weight, bias, G, eps, activation):
        codes = _dtype_codes()
        if max(shape[:2], default=0) >= 1 << 31:
            raise ValueError(f"x has shape {tuple(shape)}: images and channels are counted in 32 bits")
        if dtype not in codes:
            raise ValueError(f"x must be a float32, bfloat16 or float16 tensor on the GPU, got {dtype}")
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, got {activation!r}")
        self.layout, S, image, row = _layout_of(shape, strides, "x")
        param = dtype if weight is None and bias is None else (weight or bias)[0]
        for name, p in (("weight", weight), ("bias", bias)):
            if p is None:
                continue
            if p[0] != param or p[0] not in codes:
                raise ValueError(f"{name} must be of the other parameter's type, got {p[0]}")
            if tuple(p[1]) != (shape[1],):
                raise ValueError(f"{name} has shape {tuple(p[1])}, expected ({shape[1]},)")
        # a dense tensor like x is what torch.empty_like makes, unless x has gaps
        self.gaps = (image, row) != (shape[1] * S, S if self.layout == LAYOUT_PLANES else shape[1])
        out, dy = ((0, 0) if st is None else _layout_of(shape, st, name, self.layout)[2:]
                   for name, st in (("y", y_strides), ("dy", dy_strides)))
        self.desc = GroupNormDesc(shape[0], shape[1], G, S, self.layout, codes[dtype], codes[param],
                                  ACTIVATIONS[activation], eps, Strides(image, row), Strides(*out), Strides(*dy),
                                  Strides(0, 0))
        self.address = ctypes.addressof(self.desc)
        self.forward_bytes = oaa_group_norm_workspace_bytes(self.desc, False)
        self.backward_bytes = oaa_group_norm_workspace_bytes(self.desc, True)


_norm_call = functools.lru_cache(maxsize=4096)(_NormCall)


def _device_of(x, weight, bias):
    """The index of the one device that all are on."""
    index = x.get_device()
    if index < 0:
        raise ValueError(f"x must be a float32, bfloat16 or float16 tensor on the GPU, got {x.dtype} on {x.device}")
    for name, t in (("weight", weight), ("bias", bias)):
        if t is not None and (t.get_device() != index or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous and on {x.device}")
    return index


def _like(x, call):
    """A dense tensor of x's shape in its layout."""
    torch = _torch()[0]
    if not call.gaps:
        return torch.empty_like(x)
    if call.layout == LAYOUT_PLANES:
        return torch.empty(x.shape, dtype=x.dtype, device=x.device)
    return torch.empty((x.shape[0], *x.shape[2:], x.shape[1]), dtype=x.dtype, device=x.device).movedim(-1, 1)


def _kinds(weight, bias):
    return (None if weight is None else (weight.dtype, weight.shape),
            None if bias is None else (bias.dtype, bias.shape))


def _pointer(t):
    return None if t is None else t.data_ptr()


def _forward(call, index, x, weight, bias, y, mean, rstd):
    """The launch; mean and rstd are addresses or None."""
    need = call.forward_bytes
    ws = _torch()[0].empty(need, dtype=_torch()[0].uint8, device=x.device) if need else None
    _launch(load().oaa_group_norm_forward, index, call.address, x.data_ptr(), _pointer(weight), _pointer(bias),
            y.data_ptr(), mean, rstd, _pointer(ws), need)


def _backward(call, index, dy, x, weight, bias, mean, rstd, ws, need_x, need_weight, need_bias):
    """The launch into new tensors; mean, rstd and ws (or None) are addresses."""
    torch = _torch()[0]
    dx = _like(x, call) if need_x else None
    dweight = torch.empty_like(weight) if need_weight and weight is not None else None
    dbias = torch.empty_like(bias) if need_bias and bias is not None else None
    if dx is None and dweight is None and dbias is None:
        return None, None, None
    need = call.backward_bytes
    if need and ws is None:
        held = torch.empty(need, dtype=torch.uint8, device=x.device)  # until the launch
        ws = held.data_ptr()
    _launch(load().oaa_group_norm_backward, index, call.address, dy.data_ptr(), x.data_ptr(), _pointer(weight),
            _pointer(bias), mean, rstd, _pointer(dx), _pointer(dweight), _pointer(dbias), ws, need)
    return dx, dweight, dbias


def group_norm_forward(x, num_groups, weight=None, bias=None, eps=1e-5, activation="none", y=None, stats=True):
    """oaa_group_norm_forward on torch's current stream of x's device: (y, mean,
    rstd), the last two [B, G] float32 (None without ``stats``). x[B, C, ...]
    is laid out in planes or channels last, and so is y, whose memory x does not share."""
    torch = _torch()[0]
    index = _device_of(x, weight, bias)
    if y is not None and (y.shape != x.shape or y.dtype != x.dtype or y.get_device() != index):
        raise ValueError(f"y must be a {x.dtype} tensor of shape {tuple(x.shape)} on {x.device}")
    call = _norm_call(x.shape, x.stride(), None if y is None else y.stride(), None, x.dtype, *_kinds(weight, bias),
                      num_groups, eps, activation)
    out = _like(x, call) if y is None else y
    mean = rstd = None
    if stats:
        mean = torch.empty((x.shape[0], num_groups), dtype=torch.float32, device=x.device)
        rstd = torch.empty_like(mean)
    _forward(call, index, x, weight, bias, out, _pointer(mean), _pointer(rstd))
    if y is not None:
        _written()(y)
    return out, mean, rstd


def group_norm_backward(dy, x, num_groups, weight, bias, mean, rstd, activation="none", need_x=True, need_weight=True,
                        need_bias=True):
    """oaa_group_norm_backward on torch's current stream of x's device: (dx,
    dweight, dbias), None for each that is not needed or whose parameter is
    None. mean and rstd are the forward pass's."""
    torch = _torch()[0]
    index = _device_of(x, weight, bias)
    if dy.shape != x.shape or dy.dtype != x.dtype or dy.get_device() != index:
        raise ValueError(f"dy must be a {x.dtype} tensor of shape {tuple(x.shape)} on {x.device}")
    call = _norm_call(x.shape, x.stride(), None, dy.stride(), x.dtype, *_kinds(weight, bias), num_groups, 0.0,
                      activation)
    groups = (x.shape[0], num_groups)
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t.shape != groups or t.dtype != torch.float32 or t.get_device() != index or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 tensor of shape {groups} on {x.device}")
    return _backward(call, index, dy, x, weight, bias, mean.data_ptr(), rstd.data_ptr(), None, need_x, need_weight,
                     need_bias)


# Most bytes of backward workspace that a recorded forward pass keeps beside its
# statistics: allocating it then is cheaper than in autograd's backward thread.
_KEPT_BYTES = 1 << 20


class GroupNormRecord:
    """A forward pass whose backward pass follows, for autograd: its output y, and
    in one buffer the statistics and, if it is small, the backward workspace."""

    def __init__(self, x, num_groups, weight, bias, eps, activation):
        torch = _torch()[0]
        self.index = _device_of(x, weight, bias)
        # dy mostly comes with x's strides
        self.strides = x.stride()
        self.args = (x.dtype, *_kinds(weight, bias), num_groups, eps, activation)
        self.call = _norm_call(x.shape, self.strides, None, self.strides, *self.args)
        self.row = 4 * x.shape[0] * num_groups
        stats = (2 * self.row + 255) // 256 * 256
        self.kept = self.call.backward_bytes if self.call.backward_bytes <= _KEPT_BYTES else 0
        self.ws = stats
        self.buffer = torch.empty(stats + self.kept, dtype=torch.uint8, device=x.device)
        self.y = _like(x, self.call)
        at = self.buffer.data_ptr()
        _forward(self.call, self.index, x, weight, bias, self.y, at, at + self.row)

    def backward(self, dy, x, weight, bias, buffer, need_x, need_weight, need_bias):
        """(dx, dweight, dbias) from the tensors as autograd kept them: hooks on
        saved tensors may bring x back with other strides than it had."""
        index, C = self.index, self.call.desc.C
        if x.dtype != self.args[0] or x.shape != dy.shape:
            raise ValueError("a saved tensor came back with another type or shape")
        if x.get_device() != index or buffer.get_device() != index:
            raise ValueError(f"a saved tensor came back on another device than cuda:{index}")
        for t, kind in ((weight, self.args[1]), (bias, self.args[2])):
            if (t is None) != (kind is None) or t is not None and (
                    t.dtype != kind[0] or t.numel() != C or t.get_device() != index or not t.is_contiguous()):
                raise ValueError("a saved parameter came back with another type, shape, layout or device")
        call, at = self.call, buffer.data_ptr()
        if x.stride() != self.strides or dy.stride() != self.strides:
            call = _norm_call(x.shape, x.stride(), None, dy.stride(), *self.args)
        # another layout may need a larger workspace than was kept
        ws = at + self.ws if call.backward_bytes <= self.kept and (at + self.ws) % 256 == 0 else None
        return _backward(call, index, dy, x, weight, bias, at, at + self.row, ws, need_x, need_weight, need_bias)


NORM_TYPES = {1.0: NORM_SUM, 2.0: NORM_EUCLIDEAN, float("inf"): NORM_MAX}


def _dense(t):
    """Whether t's values fill their memory, in whatever order."""
    if t.is_contiguous():
        return True
    expect = 1
    for st, k in sorted((st, k) for st, k in zip(t.stride(), t.shape) if k != 1):
        if st != expect:
            return False
        expect *= k
    return True


def _grad_lists(grads, index):
    """Host arrays of the tensors' addresses, sizes and types."""
    codes = _dtype_codes()
    kinds = [codes.get(t.dtype) for t in grads]
    if None in kinds or not all(t.get_device() == index for t in grads):
        i = next(i for i, (t, k) in enumerate(zip(grads, kinds)) if k is None or t.get_device() != index)
        raise ValueError(f"gradient {i} must be a float32, bfloat16 or float16 tensor on cuda:{index}")
    for i, t in enumerate(grads):
        if not t.is_contiguous() and not _dense(t):
            raise ValueError(f"gradient {i} of shape {tuple(t.shape)} has gaps or overlaps (strides {t.stride()})")
    return (array.array("Q", [t.data_ptr() for t in grads]), array.array("q", [t.numel() for t in grads]),
            array.array("i", kinds))


def _grad_call(grads, norm_type):
    """The device's index, the host arrays, the norm and the workspace of a call."""
    torch, current_device, _ = _torch()
    if norm_type not in NORM_TYPES:
        raise ValueError(f"norm_type must be one of {sorted(NORM_TYPES)}, got {norm_type!r}")
    index = grads[0].get_device() if grads else current_device()
    if index < 0:
        raise ValueError(f"gradients must be on the GPU, not on {grads[0].device}")
    lists = _grad_lists(grads, index)
    device = torch.device("cuda", index)
    return (index, lists, torch.empty((), dtype=torch.float32, device=device),
            torch.empty(oaa_grad_workspace_bytes(len(grads)), dtype=torch.uint8, device=device))


def grad_norm(grads, norm_type=2.0):
    """oaa_grad_norm on torch's current stream: the norm over all values of the
    tensors, a float32 scalar on their device. norm_type: 1, 2 or infinity."""
    grads = list(grads)
    index, (src, sizes, kinds), norm, ws = _grad_call(grads, norm_type)
    _launch(load().oaa_grad_norm, index, len(grads), src.buffer_info()[0], sizes.buffer_info()[0],
            kinds.buffer_info()[0], NORM_TYPES[norm_type], norm.data_ptr(), ws.data_ptr(), ws.numel())
    return norm


def grad_clip(grads, max_norm, norm_type=2.0, out=None):
    """oaa_grad_clip on torch's current stream: the tensors scaled by min(1,
    max_norm / (norm + 1e-6)), in place or into ``out`` (tensors of the same
    shapes, types and strides that overlap neither each other nor a gradient; an
    output may be its own gradient). Returns the norm before clipping."""
    grads = list(grads)
    index, (src, sizes, kinds), norm, ws = _grad_call(grads, norm_type)
    dst = src
    if out is not None:
        out = list(out)
        if len(out) != len(grads):
            raise ValueError(f"{len(out)} outputs for {len(grads)} gradients")
        for i, (g, o) in enumerate(zip(grads, out)):
            if o.dtype != g.dtype or o.get_device() != index or o.shape != g.shape or o.stride() != g.stride():
                raise ValueError(f"output {i} differs from its gradient in shape, strides, type or device")
        dst = array.array("Q", [t.data_ptr() for t in out])
    if len(set(dst)) < len(dst):
        written = [d for d, n in zip(dst, sizes) if n]
        if len(set(written)) < len(written):
            raise ValueError("a tensor is written twice: list each gradient once")
    _launch(load().oaa_grad_clip, index, len(grads), src.buffer_info()[0], dst.buffer_info()[0],
            sizes.buffer_info()[0], kinds.buffer_info()[0], NORM_TYPES[norm_type], max_norm, norm.data_ptr(),
            ws.data_ptr(), ws.numel())
    _written()(grads if out is None else out)
    return norm
