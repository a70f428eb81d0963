"""ctypes binding of region selection, region attention and dropout: argument marshalling only.

Function names match the C ABI (include/slide_attn.h, which has the definitions).  Activations are float32 or bfloat16 tensors
[B, H, W, heads * head_dim], channels last; q, k and v may be parts of a wider tensor (a slice of the channels of one
projection's output, the first columns of a longer cache) as long as the channels of a pixel are contiguous and the pixels of an
image evenly spaced in raster order.  A sequence [B, n, C] is passed as a map of height 1.  Work is enqueued on torch's current
stream of the tensors' device.
"""
import ctypes
import functools

import torch

from .binding import SLIDE_BF16, SLIDE_F32, SlideAttnError, _check, _stream, load_library

_vp = ctypes.c_void_p
_SELECT, _FWD, _BWD = 0, 1, 2


class _Problem(ctypes.Structure):
    """slide_region_problem."""
    _fields_ = [(n, ctypes.c_int) for n in ("B", "heads", "kv_heads", "head_dim", "q_h", "q_w", "k_h", "k_w", "q_region_h",
                                            "q_region_w", "k_region_h", "k_region_w", "topk", "dtype")] + \
               [(n, ctypes.c_longlong) for n in ("q_pixel", "q_image", "k_pixel", "k_image", "v_pixel", "v_image")] + \
               [("q_size", _vp), ("k_size", _vp), ("scale", ctypes.c_float), ("dropout", ctypes.c_float),
                ("seed", ctypes.c_ulonglong), ("offset", ctypes.c_uint), ("offset_device", _vp)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        i, sz, u64, u32, ll = ctypes.c_int, ctypes.c_size_t, ctypes.c_ulonglong, ctypes.c_uint, ctypes.c_longlong
        p = ctypes.POINTER(_Problem)
        lib.slide_region_workspace_bytes.restype = sz
        lib.slide_region_workspace_bytes.argtypes = [p, i]
        lib.slide_region_select.restype = i
        lib.slide_region_select.argtypes = [p] + [_vp] * 4 + [sz, _vp]
        lib.slide_region_attn_fwd.restype = i
        lib.slide_region_attn_fwd.argtypes = [p] + [_vp] * 7 + [sz, _vp]
        lib.slide_region_attn_bwd.restype = i
        lib.slide_region_attn_bwd.argtypes = [p] + [_vp] * 11 + [sz, _vp]
        lib.slide_dropout_fwd.restype = i
        lib.slide_dropout_fwd.argtypes = [_vp] * 3 + [ll, i, ctypes.c_float, u64, u32, _vp, _vp]
        lib.slide_dropout_bwd.restype = i
        lib.slide_dropout_bwd.argtypes = [_vp] * 2 + [ll, i, ctypes.c_float, u64, u32, _vp, _vp]
        _lib = lib
    return _lib


_CODES = {torch.float32: SLIDE_F32, torch.bfloat16: SLIDE_BF16}


def _int(value, name, lo, hi):
    if isinstance(value, bool) or not hasattr(value, "__index__") or not lo <= value.__index__() <= hi:
        raise SlideAttnError("%s must be an integer in [%d, %d]" % (name, lo, hi))
    return value.__index__()


def _strides(shape, stride, name):
    """Elements between the pixels and between the images of a [B, H, W, C] tensor."""
    B, H, W, C = shape
    sb, sh, sw, sc = stride
    if W == 1:                                  # (strides of single elements say nothing)
        sw = sh if H > 1 else C
    if (C > 1 and sc != 1) or (H > 1 and sh != W * sw):
        raise SlideAttnError("%s must have contiguous channels and evenly spaced pixels" % name)
    return sw, (sb if B > 1 else 0)


def _on(t, name, device):
    if not t.is_cuda:
        raise SlideAttnError("%s must live on the GPU" % name)
    if t.device != device:
        raise SlideAttnError("%s must live on the device of the first argument" % name)


def _like(t, name, shape, dtype, device):
    """A tensor that must have this shape and type, and be contiguous."""
    if t.shape != shape or t.dtype != dtype:
        raise SlideAttnError("%s must be %s %s" % (name, str(dtype)[6:], list(shape)))
    _on(t, name, device)
    if not t.is_contiguous():
        raise SlideAttnError("%s must be contiguous" % name)
    return t.data_ptr()


def _random(dropout, seed, offset, device):
    """Rate, seed, number of the call, and where the rest of that number is read from on the device."""
    # (also as the float32 that it becomes, which may round up to the limit)
    if not 0.0 <= dropout < 1.0 - 2.0 ** -17 or ctypes.c_float(dropout).value >= 1.0 - 2.0 ** -17:
        raise SlideAttnError("dropout must be in [0, 1 - 2^-17)")
    number, holder = (0, offset) if isinstance(offset, torch.Tensor) else (_int(offset, "offset", 0, 2 ** 32 - 1), None)
    if holder is not None:
        if holder.dtype != torch.int64 or holder.numel() != 1:
            raise SlideAttnError("offset must be an integer or an int64 tensor with one element")
        _on(holder, "offset", device)
    return float(dropout), _int(seed, "seed", 0, 2 ** 64 - 1), number, None if holder is None else holder.data_ptr()


class _Plan:
    """What follows from the sizes, strides and types of a call: its problem without pointers, the shapes of lists and lse, and
    how much scratch each call needs on each device."""

    def __init__(self, dtype, q_shape, q_stride, maps, heads, q_region_h, q_region_w, k_region_h, k_region_w, kv_heads, topk):
        p = _Problem()
        if len(q_shape) != 4:
            raise SlideAttnError("activations must be [B, H, W, C]")
        if dtype not in _CODES:
            raise SlideAttnError("activations must be float32 or bfloat16, got %s" % dtype)
        p.dtype = _CODES[dtype]
        k_shape = maps[0][2]
        if max(*q_shape, *k_shape) >= 2 ** 31:          # (ctypes would keep the low 32 bits)
            raise SlideAttnError("maps must have sizes below 2^31")
        p.B, p.q_h, p.q_w, channels = q_shape
        p.heads = _int(heads, "heads", 1, 65535)
        p.kv_heads = p.heads if kv_heads is None else _int(kv_heads, "kv_heads", 1, 65535)
        if p.heads % p.kv_heads or channels % p.heads:
            raise SlideAttnError("channels must be a multiple of heads, and heads of kv_heads")
        p.head_dim = channels // p.heads
        if not 1 <= p.head_dim <= 128:
            raise SlideAttnError("head size must be 1..128")
        for name, kind, shape, stride in maps:
            if len(shape) != 4 or kind != dtype or shape[0] != p.B or shape[3] != p.kv_heads * p.head_dim or shape != k_shape:
                raise SlideAttnError("%s must be %s [%d, H, W, %d]%s" % (name, str(dtype)[6:], p.B, p.kv_heads * p.head_dim,
                                                                       "" if name == "k" else " as k is"))
        p.k_h, p.k_w = k_shape[1], k_shape[2]
        if min(p.B, p.q_h, p.q_w, p.k_h, p.k_w) < 1:
            raise SlideAttnError("maps must not be empty")
        p.q_pixel, p.q_image = _strides(q_shape, q_stride, "q")
        p.k_pixel, p.k_image = _strides(k_shape, maps[0][3], "k")
        p.v_pixel, p.v_image = _strides(k_shape, maps[1][3], "v") if len(maps) > 1 else (0, 0)
        p.q_region_h, p.q_region_w = (_int(n, "q_region", 1, 2 ** 31 - 1) for n in (q_region_h, q_region_w))
        p.k_region_h, p.k_region_w = (_int(n, "k_region", 1, 2 ** 31 - 1) for n in (k_region_h, k_region_w))
        p.topk = _int(topk, "topk", 1, 1024)
        groups = -(-p.q_h // p.q_region_h) * -(-p.q_w // p.q_region_w)
        self.image = bytes(p)
        self.sizes = (p.B, 2)
        self.lists = (p.B, p.kv_heads, groups, p.topk)
        self.lse = (p.B, p.heads, p.q_h, p.q_w)
        self.need = {}

    def problem(self, q_size, k_size, device):
        p = _Problem.from_buffer_copy(self.image)
        if q_size is not None:
            p.q_size = _like(q_size, "q_size", self.sizes, torch.int32, device)
        if k_size is not None:
            p.k_size = _like(k_size, "k_size", self.sizes, torch.int32, device)
        return p

    def scratch(self, call, workspace, like, index):
        """Pointer and bytes of the scratch: the caller's, or as much as the call needs (its tensor last).

        The need is asked for once, of the problem without what a call brings along: one that is refused needs nothing."""
        if workspace is not None:
            _on(workspace, "workspace", like.device)
            if not workspace.is_contiguous():
                raise SlideAttnError("workspace must be contiguous")
            return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace
        need = self.need.get((call, index))
        if need is None:
            need = self.need[(call, index)] = _library().slide_region_workspace_bytes(_Problem.from_buffer_copy(self.image), call)
        if need == 0:
            return None, 0, None
        workspace = like.new_empty((need,), dtype=torch.uint8)
        return workspace.data_ptr(), need, workspace


# (typed: 2.0 and True are equal to 2 and 1, but are refused)
_plan_of = functools.lru_cache(maxsize=4096, typed=True)(_Plan)


def _plan(q, maps, heads, q_region, k_region, kv_heads, topk):
    """The plan of maps q, k (and v): everything that a kernel relies on is checked once per set of sizes, the devices every time."""
    try:
        (qh, qw), (kh, kw) = q_region, k_region
    except (TypeError, ValueError):
        raise SlideAttnError("q_region and k_region must be (height, width)") from None
    return _plan_of(q.dtype, q.shape, q.stride(), tuple((n, t.dtype, t.shape, t.stride()) for n, t in maps), heads, qh, qw, kh, kw, kv_heads, topk)


def _empty(t):
    """A contiguous tensor of t's shape (empty_like takes two thirds of new_empty's time, but keeps other orders)."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _device(q, maps):
    device = q.device
    if not q.is_cuda:
        raise SlideAttnError("q must live on the GPU")
    for n, t in maps:
        if t.device != device:
            _on(t, n, device)
    return device


def _on_device(call):
    """A call that finds its first tensor's device current (switching there and back costs more than a small call)."""
    name = call.__code__.co_varnames[0]

    @functools.wraps(call)
    def enqueue(*args, **kw):
        first = args[0] if args else kw.get(name)
        if not isinstance(first, torch.Tensor) or not first.is_cuda or first.device.index == torch.cuda.current_device():
            return call(*args, **kw)                    # (what is not on a GPU is refused by the call itself)
        with torch.cuda.device(first.device):
            return call(*args, **kw)
    return enqueue


@_on_device
def _region_workspace_bytes(q, k, v, code, topk, heads, q_region, k_region, kv_heads):
    maps = (("k", k), ("v", v))
    plan = _plan(q, maps, heads, q_region, k_region, kv_heads, topk)
    return int(_library().slide_region_workspace_bytes(plan.problem(None, None, _device(q, maps)), code))


def slide_region_workspace_bytes(call, q, k, topk, heads, q_region, k_region, kv_heads=None, v=None):
    """Bytes of scratch of slide_region_select ("select"), slide_region_attn_fwd ("fwd") or slide_region_attn_bwd ("bwd").

    v: where its strides are not those of k."""
    code = {"select": _SELECT, "fwd": _FWD, "bwd": _BWD}.get(call)
    if code is None:
        raise SlideAttnError('call must be "select", "fwd" or "bwd"')
    return _region_workspace_bytes(q, k, k if v is None else v, code, topk, heads, q_region, k_region, kv_heads)


@_on_device
def slide_region_select(q, k, topk, heads, q_region, k_region, kv_heads=None, q_size=None, k_size=None, index=None, workspace=None):
    """The lists: int32 [B, kv_heads, regions of q, topk], ascending, -1 behind the last.

    q_size, k_size: int32 [B, 2] tensors, the valid height and width of every image (None: the whole map)."""
    lib = _library()
    maps = (("k", k),)
    plan = _plan(q, maps, heads, q_region, k_region, kv_heads, topk)
    device = _device(q, maps)
    p = plan.problem(q_size, k_size, device)
    if index is None:
        index = q.new_empty(plan.lists, dtype=torch.int32)
    else:
        _like(index, "index", plan.lists, torch.int32, device)
    ws, size, keep = plan.scratch(_SELECT, workspace, q, device.index)
    _check(lib.slide_region_select(p, q.data_ptr(), k.data_ptr(), index.data_ptr(), ws, size, _stream(device.index)))
    return index


def _attention(q, k, v, index, heads, q_region, k_region, kv_heads, q_size, k_size, scale, dropout, seed, offset):
    """The plan, the problem with its pointers, and the lists of an attention call."""
    if index.dim() != 4:
        raise SlideAttnError("index must be int32 [B, kv_heads, regions of q, topk]")
    maps = (("k", k), ("v", v))
    plan = _plan(q, maps, heads, q_region, k_region, kv_heads, index.shape[3])
    # (as the float32 that it becomes: one too small for that would turn into 0, which stands for the default)
    if scale is not None and not 0.0 < ctypes.c_float(scale).value < float("inf"):
        raise SlideAttnError("scale must be positive in float32")
    device = _device(q, maps)
    p = plan.problem(q_size, k_size, device)
    p.dropout, p.seed, p.offset, p.offset_device = _random(dropout, seed, offset, device)
    if scale is not None:
        p.scale = scale
    return plan, p, _like(index, "index", plan.lists, torch.int32, device)


@_on_device
def slide_region_attn_fwd(q, k, v, index, heads, q_region, k_region, kv_heads=None, q_size=None, k_size=None, scale=None,
                          dropout=0.0, seed=0, offset=0, out=None, lse=None, workspace=None):
    """out: every row of q over the keys of its region's list.  lse: optional float32 [B, heads, H, W] tensor that receives
    the log of the softmax denominators (the backward takes it).

    dropout, seed, offset: of the attention weights; offset may be an int64 tensor with one element, read when the kernels run."""
    lib = _library()
    plan, p, lists = _attention(q, k, v, index, heads, q_region, k_region, kv_heads, q_size, k_size, scale, dropout, seed, offset)
    device = q.device
    if out is None:
        out = _empty(q)
    else:
        _like(out, "out", q.shape, q.dtype, device)
    lse_at = None if lse is None else _like(lse, "lse", plan.lse, torch.float32, device)
    ws, size, keep = plan.scratch(_FWD, workspace, q, device.index)
    _check(lib.slide_region_attn_fwd(p, q.data_ptr(), k.data_ptr(), v.data_ptr(), lists, out.data_ptr(), lse_at, ws, size,
                                     _stream(device.index)))
    return out


@_on_device
def slide_region_attn_bwd(dout, q, k, v, index, out, lse, heads, q_region, k_region, kv_heads=None, q_size=None, k_size=None,
                          scale=None, dropout=0.0, seed=0, offset=0, outputs=None, workspace=None):
    """Returns (dq, dk, dv), contiguous.  out, lse: the forward's results for the same arguments."""
    lib = _library()
    plan, p, lists = _attention(q, k, v, index, heads, q_region, k_region, kv_heads, q_size, k_size, scale, dropout, seed, offset)
    device = q.device
    dq, dk, dv = (_empty(q), _empty(k), _empty(v)) if outputs is None else outputs
    at = [_like(t, name, like.shape, q.dtype, device)
          for t, name, like in ((dout, "dout", q), (out, "out", q), (dq, "dq", q), (dk, "dk", k), (dv, "dv", k))]
    lse_at = _like(lse, "lse", plan.lse, torch.float32, device)
    ws, size, keep = plan.scratch(_BWD, workspace, q, device.index)
    _check(lib.slide_region_attn_bwd(p, at[0], q.data_ptr(), k.data_ptr(), v.data_ptr(), lists, at[1], lse_at, *at[2:], ws, size,
                                     _stream(device.index)))
    return dq, dk, dv


def _dropout(entry, x, name, residual, p, seed, offset, y):
    """entry's call: x, residual (False: it takes none), y, ..."""
    if not x.is_cuda:
        raise SlideAttnError("%s must live on the GPU" % name)
    if not x.is_contiguous():
        raise SlideAttnError("%s must be contiguous" % name)
    code = _CODES.get(x.dtype)
    if code is None:
        raise SlideAttnError("%s must be float32 or bfloat16, got %s" % (name, x.dtype))
    device = x.device
    p, seed, number, holder = _random(p, seed, offset, device)
    if y is None:
        y = torch.empty_like(x)
    else:
        _like(y, "the result", x.shape, x.dtype, device)
    at = (y.data_ptr(),)
    if residual is not False:
        at = (None if residual is None else _like(residual, "residual", x.shape, x.dtype, device),) + at
    if x.numel():
        _check(entry(x.data_ptr(), *at, x.numel(), code, p, seed, number, holder, _stream(device.index)))
    return y


@_on_device
def slide_dropout_fwd(x, p, seed, offset=0, residual=None, out=None):
    """residual + dropout(x) of any contiguous tensor; the mask follows from seed, offset and the element's number."""
    return _dropout(_library().slide_dropout_fwd, x, "x", residual, p, seed, offset, out)


@_on_device
def slide_dropout_bwd(dout, p, seed, offset=0, dx=None):
    """The gradient of x (the residual's is dout itself), with the mask of the forward's p, seed and offset."""
    return _dropout(_library().slide_dropout_bwd, dout, "dout", False, p, seed, offset, dx)
