"""ctypes binding of libgspc.so: argument marshalling only (in C, csrc/pycall.c, for the call that a program makes
for every layer).

Function names and argument order mirror include/gspc.h.  Device buffers are
torch tensors (PyTorch is used for device memory and streams, nothing else);
every computation runs in the library's HIP kernels.  There is no CPU
fallback: if the library is missing or a call fails, an exception is raised.
"""
import ctypes
import os
import threading

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libgspc.so")

GSPC_F32, GSPC_BF16, GSPC_I8 = 0, 1, 2
PATH_AUTO, PATH_DIRECT, PATH_MFMA = -1, 0, 1
OP_CONV, OP_MAXPOOL, OP_ADD, OP_RELU = 0, 1, 2, 3
FLAG_RELU = 1
ACT_NONE, ACT_RELU, ACT_SILU = 0, 1, 2

ERROR_NAMES = {0: "GSPC_OK", -1: "GSPC_ERR_NULL", -2: "GSPC_ERR_DIM", -3: "GSPC_ERR_GROUPS",
               -4: "GSPC_ERR_DTYPE", -5: "GSPC_ERR_MISMATCH", -6: "GSPC_ERR_SPACE",
               -7: "GSPC_ERR_HIP", -8: "GSPC_ERR_ARG"}

EXPORTS = [
    "gspc_version", "gspc_set_stream", "gspc_last_error", "gspc_output_dims", "gspc_layer_macs",
    "gspc_packed_weight_bytes", "gspc_pack_weights", "gspc_unpack_weights", "gspc_packed_free",
    "gspc_packed_info", "gspc_pack_input_bf16", "gspc_conv2d_grouped", "gspc_force_path",
    "gspc_last_path", "gspc_last_kernel", "gspc_set_graph_mode", "gspc_set_chain_fusion", "gspc_set_winograd", "gspc_run_layer_chain",
    "gspc_rows8_pitch", "gspc_pack_channels_last", "gspc_unpack_channels_last", "gspc_quantize_rows", "gspc_dequantize_rows",
    "gspc_group_norm_workspace_bytes", "gspc_group_norm_backward_workspace_bytes", "gspc_group_norm", "gspc_group_norm_backward", "gspc_matmul_i8",
]


class GspcError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"{ERROR_NAMES.get(code, code)}: {message}")
        self.code = code


class GspcLayer(ctypes.Structure):
    _fields_ = [("op", ctypes.c_int), ("src", ctypes.c_int), ("src2", ctypes.c_int),
                ("dst", ctypes.c_int), ("N", ctypes.c_int), ("Cin", ctypes.c_int),
                ("H", ctypes.c_int), ("W", ctypes.c_int), ("Cout", ctypes.c_int),
                ("KH", ctypes.c_int), ("KW", ctypes.c_int), ("stride", ctypes.c_int),
                ("pad", ctypes.c_int), ("groups", ctypes.c_int), ("flags", ctypes.c_int),
                ("w", ctypes.c_void_p)]


_thread = threading.local()     # stream: the library's, as gspc_set_stream was last given it
_lib = None
_conv = None     # gspc_conv2d_grouped through _gspc_call, or _no_conv
_fast = None     # _gspc_call with the channels-last operators, or _NoFast


def _no_conv(*args):
    """Every call of gspc_conv2d_grouped is one that only ctypes converts."""
    return NotImplemented


class _NoFast:
    """Every call of a channels-last operator is one that only ctypes converts."""
    pack = unpack = quantize = dequantize = norm = norm_backward = matmul = staticmethod(_no_conv)


def load():
    """Loads libgspc.so (must have been built in-tree) and sets prototypes."""
    global _lib, _conv, _fast
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2006_09791_amd.build` "
            "(there is no fallback path)")
    # torch first: it brings the HIP runtime whose streams and allocations are
    # handed to the library, and libgspc.so must bind to that same runtime.
    import torch
    lib = ctypes.CDLL(LIB_PATH)
    i, vp, sz = ctypes.c_int, ctypes.c_void_p, ctypes.c_size_t
    ip = ctypes.POINTER(ctypes.c_int)
    lib.gspc_version.restype = i
    lib.gspc_set_stream.restype = i
    lib.gspc_set_stream.argtypes = [vp]
    lib.gspc_last_error.restype = ctypes.c_char_p
    lib.gspc_output_dims.restype = i
    lib.gspc_output_dims.argtypes = [i] * 6 + [ip, ip]
    lib.gspc_layer_macs.restype = ctypes.c_uint64
    lib.gspc_layer_macs.argtypes = [i] * 8
    lib.gspc_packed_weight_bytes.restype = sz
    lib.gspc_packed_weight_bytes.argtypes = [i] * 6
    lib.gspc_pack_weights.restype = i
    lib.gspc_pack_weights.argtypes = [vp] + [i] * 6 + [vp, sz, ctypes.POINTER(vp)]
    lib.gspc_unpack_weights.restype = i
    lib.gspc_unpack_weights.argtypes = [vp, i, vp]
    lib.gspc_packed_free.restype = None
    lib.gspc_packed_free.argtypes = [vp]
    lib.gspc_packed_info.restype = i
    lib.gspc_packed_info.argtypes = [vp] + [ip] * 7
    lib.gspc_pack_input_bf16.restype = i
    lib.gspc_pack_input_bf16.argtypes = [vp, sz, vp]
    lib.gspc_conv2d_grouped.restype = i
    lib.gspc_conv2d_grouped.argtypes = [vp, vp] + [i] * 10 + [vp]
    lib.gspc_force_path.restype = i
    lib.gspc_force_path.argtypes = [i]
    lib.gspc_last_path.restype = i
    lib.gspc_set_graph_mode.restype = i
    lib.gspc_set_graph_mode.argtypes = [i]
    lib.gspc_set_chain_fusion.restype = i
    lib.gspc_set_chain_fusion.argtypes = [i]
    lib.gspc_set_winograd.restype = i
    lib.gspc_set_winograd.argtypes = [i]
    lib.gspc_last_kernel.restype = ctypes.c_char_p
    lib.gspc_run_layer_chain.restype = i
    lib.gspc_run_layer_chain.argtypes = [ctypes.POINTER(GspcLayer), i, ctypes.POINTER(vp),
                                         ctypes.POINTER(sz), i, ctypes.POINTER(ctypes.c_float)]
    ll, f = ctypes.c_int64, ctypes.c_float
    lib.gspc_rows8_pitch.restype = i
    lib.gspc_rows8_pitch.argtypes = [i]
    lib.gspc_pack_channels_last.restype = lib.gspc_unpack_channels_last.restype = i
    lib.gspc_pack_channels_last.argtypes = lib.gspc_unpack_channels_last.argtypes = [vp] + [i] * 4 + [vp, i]
    lib.gspc_quantize_rows.restype = i
    lib.gspc_quantize_rows.argtypes = [vp, i, ll, ll, i, vp, vp]
    lib.gspc_dequantize_rows.restype = i
    lib.gspc_dequantize_rows.argtypes = [vp, vp, ll, i, vp, i, ll]
    lib.gspc_group_norm_workspace_bytes.restype = lib.gspc_group_norm_backward_workspace_bytes.restype = sz
    lib.gspc_group_norm_workspace_bytes.argtypes = lib.gspc_group_norm_backward_workspace_bytes.argtypes = [i] * 6
    lib.gspc_group_norm.restype = i
    lib.gspc_group_norm.argtypes = [vp, i, ll, vp, vp, i, i, i, i, f, i, vp, i, ll, vp, vp, vp, vp, vp, sz]
    lib.gspc_group_norm_backward.restype = i
    lib.gspc_group_norm_backward.argtypes = [vp, i, ll, vp, i, ll, vp, vp, vp, vp, i, i, i, i, i, vp, ll, vp, vp, vp, sz]
    lib.gspc_matmul_i8.restype = i
    lib.gspc_matmul_i8.argtypes = [vp, vp, vp, vp, vp, ll, i, i, vp, i, ll]
    try:
        from . import _gspc_call
    except ImportError:          # not built for this interpreter
        _conv, _fast = _no_conv, _NoFast
    else:
        _gspc_call.bind(ctypes.cast(lib.gspc_conv2d_grouped, vp).value)
        _gspc_call.bind_tokens(*[ctypes.cast(f, vp).value for f in (
            lib.gspc_pack_channels_last, lib.gspc_unpack_channels_last, lib.gspc_quantize_rows, lib.gspc_dequantize_rows, lib.gspc_group_norm,
            lib.gspc_group_norm_backward, lib.gspc_matmul_i8)], torch.float32, torch.bfloat16, torch.int8)
        _conv, _fast = _gspc_call.conv, _gspc_call
    _lib = lib
    return lib


def _check(rc):
    if rc != 0:
        raise GspcError(rc, load().gspc_last_error().decode())


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def gspc_version():
    return load().gspc_version()


def gspc_last_error():
    return load().gspc_last_error().decode()


def gspc_set_stream(stream=None):
    """stream: torch.cuda.Stream, raw handle, or None for torch's current stream."""
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    handle = getattr(stream, "cuda_stream", stream)
    _check(load().gspc_set_stream(ctypes.c_void_p(handle)))
    _thread.stream = handle or 0


def gspc_output_dims(H, W, KH, KW, stride, pad):
    ho, wo = ctypes.c_int(), ctypes.c_int()
    _check(load().gspc_output_dims(H, W, KH, KW, stride, pad, ctypes.byref(ho), ctypes.byref(wo)))
    return ho.value, wo.value


def gspc_layer_macs(N, Cin, Cout, KH, KW, Hout, Wout, groups):
    return int(load().gspc_layer_macs(N, Cin, Cout, KH, KW, Hout, Wout, groups))


def gspc_packed_weight_bytes(Cin, Cout, KH, KW, groups, dtype=GSPC_F32):
    n = load().gspc_packed_weight_bytes(Cin, Cout, KH, KW, groups, dtype)
    if n == 0:
        raise GspcError(-8, gspc_last_error())
    return int(n)


class PackedWeights:
    """Owns the device bytes (a torch uint8 tensor) and the host descriptor."""

    def __init__(self, handle, storage, Cin, Cout, KH, KW, groups, dtype):
        self.handle, self.storage = handle, storage
        self.Cin, self.Cout, self.KH, self.KW, self.groups, self.dtype = Cin, Cout, KH, KW, groups, dtype

    def info(self):
        vals = [ctypes.c_int() for _ in range(7)]
        _check(load().gspc_packed_info(self.handle, *[ctypes.byref(v) for v in vals]))
        keys = ["Cin", "Cout", "KH", "KW", "groups", "dtype", "has_mfma"]
        return dict(zip(keys, (v.value for v in vals)))

    def free(self):
        if self.handle:
            load().gspc_packed_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def gspc_pack_weights(weight, groups, dtype=GSPC_F32):
    """weight: fp32 CUDA tensor [Cout, Cin/g, KH, KW] -> PackedWeights."""
    import torch
    assert weight.is_cuda and weight.dtype == torch.float32 and weight.is_contiguous()
    Cout, CPG, KH, KW = weight.shape
    Cin = CPG * groups
    nbytes = gspc_packed_weight_bytes(Cin, Cout, KH, KW, groups, dtype)
    storage = torch.empty(nbytes + 256, dtype=torch.uint8, device=weight.device)
    off = (-storage.data_ptr()) % 256
    handle = ctypes.c_void_p()
    _check(load().gspc_pack_weights(_ptr(weight), Cin, Cout, KH, KW, groups, dtype,
                                    ctypes.c_void_p(storage.data_ptr() + off), nbytes,
                                    ctypes.byref(handle)))
    return PackedWeights(handle, storage, Cin, Cout, KH, KW, groups, dtype)


def gspc_unpack_weights(packed, which=PATH_DIRECT):
    import torch
    out = torch.empty((packed.Cout, packed.Cin // packed.groups, packed.KH, packed.KW),
                      dtype=torch.float32, device=packed.storage.device)
    _check(load().gspc_unpack_weights(packed.handle, which, _ptr(out)))
    return out


def gspc_pack_input_bf16(x):
    """fp32 CUDA tensor -> bf16 CUDA tensor of the same shape (library kernel)."""
    import torch
    assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous()
    out = torch.empty(x.shape, dtype=torch.bfloat16, device=x.device)
    _check(load().gspc_pack_input_bf16(_ptr(x), x.numel(), _ptr(out)))
    return out


def gspc_conv2d_grouped(input, packed_weight, N, Cin, H, W, Cout, KH, KW, stride, pad, groups,
                        output=None):
    """Returns the fp32 output tensor [N, Cout, Hout, Wout] (allocated if not given)."""
    if _lib is None:
        load()
    if output is None:
        import torch
        ho, wo = gspc_output_dims(H, W, KH, KW, stride, pad)
        output = torch.empty((N, Cout, ho, wo), dtype=torch.float32, device=input.device)
    rc = _conv(input, packed_weight.handle, N, Cin, H, W, Cout, KH, KW, stride, pad, groups, output)
    if rc is NotImplemented:
        rc = _lib.gspc_conv2d_grouped(_ptr(input), packed_weight.handle, N, Cin, H, W, Cout, KH, KW, stride, pad, groups,
                                      _ptr(output))
    if rc:
        _check(rc)
    return output


def gspc_force_path(path):
    _check(load().gspc_force_path(path))


def gspc_set_graph_mode(on):
    _check(load().gspc_set_graph_mode(1 if on else 0))


def gspc_set_chain_fusion(on):
    _check(load().gspc_set_chain_fusion(1 if on else 0))


def gspc_set_winograd(on):
    """on: True / 1 = every eligible layer, False / 0 = never, None / -1 = automatic (default)."""
    _check(load().gspc_set_winograd(-1 if on is None or (on is not True and on < 0) else (1 if on else 0)))


def gspc_last_path():
    return load().gspc_last_path()


def gspc_last_kernel():
    return load().gspc_last_kernel().decode()


class LayerChain:
    """Marshalled form of a list of workloads.Layer: C layer array, buffer table."""

    def __init__(self, layers, packed, buffers):
        """layers: list of workloads.Layer; packed: PackedWeights indexed by
        Layer.wid; buffers: CUDA tensors indexed by the layers' src/src2/dst."""
        ops = {"conv": OP_CONV, "maxpool": OP_MAXPOOL, "add": OP_ADD, "relu": OP_RELU}
        self.n_layers = len(layers)
        self.layers = (GspcLayer * self.n_layers)()
        for k, l in enumerate(layers):
            g = self.layers[k]
            g.op, g.src, g.src2, g.dst = ops[l.op], l.src, l.src2, l.dst
            g.N, g.Cin, g.H, g.W, g.Cout = l.N, l.Cin, l.H, l.W, l.Cout
            g.KH, g.KW, g.stride, g.pad, g.groups = l.KH, l.KW, l.stride, l.pad, l.groups
            g.flags = FLAG_RELU if l.relu else 0
            g.w = packed[l.wid].handle.value if l.op == "conv" else None
        self.keep = (packed, buffers)
        self.n_bufs = len(buffers)
        self.bufs = (ctypes.c_void_p * self.n_bufs)(*[b.data_ptr() for b in buffers])
        self.bytes = (ctypes.c_size_t * self.n_bufs)(*[b.numel() * b.element_size() for b in buffers])


def gspc_run_layer_chain(lc, per_layer_ms=False):
    ms = (ctypes.c_float * lc.n_layers)() if per_layer_ms else None
    _check(load().gspc_run_layer_chain(lc.layers, lc.n_layers, lc.bufs, lc.bytes, lc.n_bufs, ms))
    return list(ms) if per_layer_ms else None


# ---- channels-last operators -------------------------------------------------------------------
# Tokens are torch tensors [..., channels] whose rows are a fixed distance apart (a contiguous tensor, or a slice of the
# channels of one); 8-bit rows are a pair (int8 tensor [rows, pitch], fp32 scales [rows]).

def _empty(shape, dtype, device):
    """A tensor for the library's stream: torch reuses its memory after work of that stream only."""
    import torch
    stream = getattr(_thread, "stream", 0)
    if stream == _current_stream(device):
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)):
        return torch.empty(shape, dtype=dtype, device=device)


def _current_stream(device):
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)      # a twentieth of the time of a Stream object
    return raw(device.index) if raw is not None and device.index is not None else torch.cuda.current_stream(device).cuda_stream


_DTYPES = {}


def _dtypes():
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.float32: GSPC_F32, torch.bfloat16: GSPC_BF16})
    return _DTYPES


def _dtype(t, what):
    kind = _dtypes().get(t.dtype)
    if kind is None:
        raise GspcError(-4, f"{what}: {t.dtype} is neither float32 nor bfloat16")
    return kind


def _torch_dtype(dtype):
    for t, kind in _dtypes().items():
        if kind == dtype:
            return t
    raise GspcError(-4, f"unknown dtype {dtype}")


def _on_gpu(t, what):
    if not t.is_cuda:
        raise GspcError(-8, f"{what} is not on the GPU")
    return t


def _row_stride(t, what):
    """Elements between two rows of t's last dimension."""
    _on_gpu(t, what)
    if t.is_contiguous():
        return t.shape[-1]
    shape, stride = t.shape, t.stride()
    if len(shape) < 2 or (stride[-1] != 1 and shape[-1] > 1):
        raise GspcError(-8, f"{what}: channels must be side by side")
    ld, step = None, None
    for k in range(len(shape) - 2, -1, -1):
        if shape[k] == 1:
            continue
        if ld is None:
            ld = step = stride[k]
        if stride[k] != step:
            raise GspcError(-8, f"{what}: rows must be a fixed distance apart")
        step *= shape[k]
    return shape[-1] if ld is None else ld


def _flat(t, dtype, count, what):
    """A contiguous tensor of that type and number of elements, or None."""
    if t is None:
        return None
    _on_gpu(t, what)
    if t.dtype != dtype or t.numel() != count or not t.is_contiguous():
        raise GspcError(-8, f"{what}: a contiguous {dtype} tensor of {count} elements is needed")
    return t.data_ptr()


def _rows8(pair, rows, cols, what):
    import torch
    q, scale = pair
    return (_flat(q, torch.int8, rows * gspc_rows8_pitch(cols), what), _flat(scale, torch.float32, rows, what + " scales"))


def _same_shape(t, shape, what):
    if tuple(t.shape) != tuple(shape):
        raise GspcError(-2, f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def gspc_rows8_pitch(cols):
    if cols <= 0 or cols > 0x7ffffff0:
        raise GspcError(-2, f"{cols} columns")
    return (cols + 15) // 16 * 16


def _new_rows8(rows, cols, device):
    import torch
    return (_empty((rows, gspc_rows8_pitch(cols)), torch.int8, device), _empty((rows,), torch.float32, device))


def _done(rc):
    """Whether the call through _gspc_call was made; its error is raised."""
    if rc is NotImplemented:
        return False
    if rc:
        _check(rc)
    return True


def _change_layout(call, x, out, dtype, pack):
    _on_gpu(x, "x")
    if x.dim() < 3 or not x.is_contiguous():
        raise GspcError(-8, "x: a contiguous tensor of images, channels and pixels is needed")
    N = x.shape[0]
    C = x.shape[1] if pack else x.shape[-1]
    P = 1
    for n in x.shape[2:] if pack else x.shape[1:-1]:
        P *= n
    shape = (N, P, C) if pack else (N, C, P)
    if out is None:
        out = _empty(shape, _torch_dtype(dtype), x.device)
    elif not ((out.dim() >= 3 and out.shape[0] == N and out.shape[-1 if pack else 1] == C and out.numel() == x.numel())
              or (pack and tuple(out.shape) == (N * P, C))):
        raise GspcError(-2, f"out has shape {tuple(out.shape)}, expected {shape}, with its pixels in one dimension or more")
    elif not _on_gpu(out, "out").is_contiguous():
        raise GspcError(-8, "out must be contiguous")
    _check(call(x.data_ptr(), _dtype(x, "x"), N, C, P, out.data_ptr(), _dtype(out, "out")))
    return out


def gspc_pack_channels_last(x, out=None, dtype=GSPC_BF16):
    """x [N, C, ...] (planes) -> [N, P, C] (tokens), P the pixels of a plane; `out`: a tensor [N, ..., C] or [N * P, C] to write into."""
    if out is not None and _fast is not None and _done(_fast.pack(x, out)):
        return out
    return _change_layout(load().gspc_pack_channels_last, x, out, dtype, True)


def gspc_unpack_channels_last(x, out=None, dtype=GSPC_F32):
    """x [N, ..., C] (tokens) -> [N, C, P] (planes); `out`: a tensor [N, C, ...] to write into."""
    if out is not None and _fast is not None and _done(_fast.unpack(x, out)):
        return out
    return _change_layout(load().gspc_unpack_channels_last, x, out, dtype, False)


def gspc_quantize_rows(x, out=None):
    """x [..., cols] -> 8-bit rows (q [rows, pitch], scale [rows]); `out`: such a pair to write into."""
    if out is not None and _fast is not None and _done(_fast.quantize(x, out)):
        return out
    lib = load()
    ld, cols = _row_stride(x, "x"), x.shape[-1]
    if cols == 0:
        raise GspcError(-2, "x has no columns")
    rows = x.numel() // cols
    if out is None:
        out = _new_rows8(rows, cols, x.device)
    q, scale = _rows8(out, rows, cols, "out")
    _check(lib.gspc_quantize_rows(x.data_ptr(), _dtype(x, "x"), ld, rows, cols, q, scale))
    return out


def gspc_dequantize_rows(rows8, cols, out=None, dtype=GSPC_F32):
    """8-bit rows of `cols` values -> [rows, cols]; `out`: a tensor [..., cols] to write into."""
    if out is not None and _fast is not None and _done(_fast.dequantize(rows8, cols, out)):
        return out
    lib = load()
    rows = rows8[1].numel()
    q, scale = _rows8(rows8, rows, cols, "rows8")
    if out is None:
        out = _empty((rows, cols), _torch_dtype(dtype), rows8[0].device)
    elif out.shape[-1] != cols or out.numel() != rows * cols:
        raise GspcError(-2, f"out has shape {tuple(out.shape)}, expected {rows} rows of {cols}")
    _check(lib.gspc_dequantize_rows(q, scale, rows, cols, out.data_ptr(), _dtype(out, "out"), _row_stride(out, "out")))
    return out


def gspc_group_norm_workspace_bytes(N, P, C, groups, x_dtype, rows8=False):
    return int(load().gspc_group_norm_workspace_bytes(N, P, C, groups, x_dtype, 1 if rows8 else 0))


def gspc_group_norm_backward_workspace_bytes(N, P, C, groups, dy_dtype, x_dtype):
    return int(load().gspc_group_norm_backward_workspace_bytes(N, P, C, groups, dy_dtype, x_dtype))


def _tokens(x, what):
    if _on_gpu(x, what).dim() < 3:
        raise GspcError(-2, f"{what}: [images, pixels, channels] is needed")
    N, C, P = x.shape[0], x.shape[-1], 1
    for n in x.shape[1:-1]:
        P *= n
    return N, P, C


def _scratch(nbytes, device):
    import torch
    return _empty((nbytes,), torch.int8, device)


def _workspace(workspace, need, device):
    """(address, bytes) of the caller's workspace, or of one of `need` bytes, and the tensor behind it."""
    if workspace is None:
        if not need:
            return None, 0, None
        workspace = _scratch(need, device)
    elif not _on_gpu(workspace, "workspace").is_contiguous():
        raise GspcError(-8, "workspace must be contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def gspc_group_norm(x, gamma, beta, groups, eps=1e-5, act=ACT_NONE, out=None, dtype=None, stats=None, saved=None, workspace=None):
    """x [N, ..., C] -> y of x's shape (type: `dtype`, by default x's), or 8-bit rows of it where `dtype` is GSPC_I8 or `out` is
    a pair.  stats: fp32 [N, groups, 2] to write mean and 1 / sqrt(var + eps) to; saved: 8-bit rows to write x to."""
    if out is not None and _fast is not None:
        rc = _fast.norm(x, gamma, beta, groups, eps, act, out, stats, saved, workspace)
        if rc == -6 and workspace is None:  # GSPC_ERR_SPACE: a call that needs one
            N, P, C = _tokens(x, "x")
            need = gspc_group_norm_workspace_bytes(N, P, C, groups, _dtype(x, "x"), isinstance(out, (tuple, list)) or saved is not None)
            rc = _fast.norm(x, gamma, beta, groups, eps, act, out, stats, saved, _scratch(need, x.device))
        if _done(rc):
            return out
    import torch
    lib = load()
    N, P, C = _tokens(x, "x")
    if out is None:
        out = _new_rows8(N * P, C, x.device) if dtype == GSPC_I8 else _empty(x.shape, x.dtype if dtype is None else _torch_dtype(dtype), x.device)
    if isinstance(out, (tuple, list)):
        (y, y_scale), kind, ldy = _rows8(out, N * P, C, "out"), GSPC_I8, 0
    else:
        _same_shape(out, x.shape, "out")
        y, y_scale, kind, ldy = out.data_ptr(), None, _dtype(out, "out"), _row_stride(out, "out")
    q, scale = (None, None) if saved is None else _rows8(saved, N * P, C, "saved")
    x_kind = _dtype(x, "x")
    ws, ws_bytes, held = _workspace(workspace, workspace is None and gspc_group_norm_workspace_bytes(
        N, P, C, groups, x_kind, kind == GSPC_I8 or saved is not None), x.device)
    _check(lib.gspc_group_norm(x.data_ptr(), x_kind, _row_stride(x, "x"), _flat(gamma, torch.float32, C, "gamma"),
                               _flat(beta, torch.float32, C, "beta"), N, P, C, groups, eps, act, y, kind, ldy, y_scale,
                               _flat(stats, torch.float32, N * groups * 2, "stats"), q, scale, ws, ws_bytes))
    return out


def gspc_group_norm_backward(dy, x, stats, gamma, beta, groups, act=ACT_NONE, dx=None, dgamma=None, dbeta=None, workspace=None):
    """dy [N, ..., C], x of its shape or 8-bit rows of it -> (dx, dgamma, dbeta), dx of dy's type."""
    if dx is not None and dgamma is not None and dbeta is not None and _fast is not None:
        rc = _fast.norm_backward(dy, x, stats, gamma, beta, groups, act, dx, dgamma, dbeta, workspace)
        if rc == -6 and workspace is None:  # GSPC_ERR_SPACE: a call that needs one
            N, P, C = _tokens(dy, "dy")
            need = gspc_group_norm_backward_workspace_bytes(N, P, C, groups, _dtype(dy, "dy"), GSPC_I8 if isinstance(x, (tuple, list)) else _dtype(x, "x"))
            rc = _fast.norm_backward(dy, x, stats, gamma, beta, groups, act, dx, dgamma, dbeta, _scratch(need, dy.device))
        if _done(rc):
            return dx, dgamma, dbeta
    import torch
    lib = load()
    N, P, C = _tokens(dy, "dy")
    if isinstance(x, (tuple, list)):
        (px, x_scale), kind, ldx = _rows8(x, N * P, C, "x"), GSPC_I8, 0
    else:
        _same_shape(x, dy.shape, "x")
        px, x_scale, kind, ldx = x.data_ptr(), None, _dtype(x, "x"), _row_stride(x, "x")
    if dx is None:
        dx = _empty(dy.shape, dy.dtype, dy.device)
    _same_shape(dx, dy.shape, "dx")
    if dx.dtype != dy.dtype:
        raise GspcError(-4, f"dx is {dx.dtype}, dy {dy.dtype}")
    if dgamma is None:
        dgamma = _empty((C,), torch.float32, dy.device)
    if dbeta is None:
        dbeta = _empty((C,), torch.float32, dy.device)
    dy_kind = _dtype(dy, "dy")
    ws, ws_bytes, held = _workspace(workspace, workspace is None and gspc_group_norm_backward_workspace_bytes(
        N, P, C, groups, dy_kind, kind), dy.device)
    _check(lib.gspc_group_norm_backward(dy.data_ptr(), dy_kind, _row_stride(dy, "dy"), px, kind, ldx, x_scale,
                                        _flat(stats, torch.float32, N * groups * 2, "stats"), _flat(gamma, torch.float32, C, "gamma"),
                                        _flat(beta, torch.float32, C, "beta"), N, P, C, groups, act, dx.data_ptr(), _row_stride(dx, "dx"),
                                        _flat(dgamma, torch.float32, C, "dgamma"), _flat(dbeta, torch.float32, C, "dbeta"),
                                        ws, ws_bytes))
    return dx, dgamma, dbeta


def gspc_matmul_i8(a, w, bias=None, out=None, dtype=GSPC_BF16, cols=None):
    """8-bit rows a (M tokens) and w (N filters) of the same length -> [M, N]; `out`: a tensor [..., N] to write into.  cols: that
    length, checked against both; without it all of the rows' pitch is summed, whose padding is zero (rows of 133137 to 133144 values,
    the longest there are, have a longer pitch than may be summed, and need it)."""
    if out is not None and _fast is not None and _done(_fast.matmul(a, w, bias, out, cols)):
        return out
    import torch
    lib = load()
    K, M, N = a[0].shape[-1], a[1].numel(), w[1].numel()
    if w[0].shape[-1] != K:
        raise GspcError(-5, f"tokens of {K} values, filters of {w[0].shape[-1]}")
    if cols is not None:
        if gspc_rows8_pitch(cols) != K:
            raise GspcError(-5, f"rows of {cols} values have a pitch of {gspc_rows8_pitch(cols)}, these of {K}")
        K = cols
    qa, sa = _rows8(a, M, K, "a")
    qw, sw = _rows8(w, N, K, "w")
    if out is None:
        out = _empty((M, N), _torch_dtype(dtype), a[0].device)
    elif out.shape[-1] != N or out.numel() != M * N:
        raise GspcError(-2, f"out has shape {tuple(out.shape)}, expected {M} rows of {N}")
    _check(lib.gspc_matmul_i8(qa, sa, qw, sw, _flat(bias, torch.float32, N, "bias"), M, N, K, out.data_ptr(), _dtype(out, "out"),
                              _row_stride(out, "out")))
    return out
