"""Binding of the operators of a rectified feed-forward block.

    n = isc_rmsnorm(x, w, residual=r, mx8=True)        # n.h, n.mx8
    r = isc_route(logits, 8, score="sigmoid")          # r.ids, r.weights, r.offsets, r.order
    u = isc_w4_linear(n.mx8, up, route=r, relu=True)   # [T, 8, F], most of it zeros
    y = isc_w4_skip(u, down, route=r)                  # [T, D], the zeros of u skipped

Argument marshalling only, as in the package itself; the C functions' names
and rules (include/isc.h) are these functions'.  Leading dimensions of a tensor
count as rows; a tensor whose rows are not evenly spaced, or whose values
within a row are not consecutive, is copied first.  Tensors live on the current
device.  Outputs and workspaces are allocated on the stream of the call.
"""
from __future__ import annotations

import ctypes
import functools
import inspect
from typing import NamedTuple

import paper_1704_07724_amd as _isc

F32, F16, BF16, MX8 = 0, 1, 2, 3
SCORES = {"softmax": 0, "sigmoid": 1}
LAYOUTS = {"tiles": 0, "rows": 1}
# Tokens that fill one matrix operand, by type: isc_w4_linear has a workspace for more, and
# none for up to a third of them.
COLUMNS = {F32: 5, F16: 8, BF16: 16, MX8: 16}


class W4Desc(ctypes.Structure):
    """isc_w4_desc: E matrices of N outputs x K inputs, and their layout."""
    _fields_ = [(n, ctypes.c_int32) for n in ("E", "N", "K", "layout")]


class Mx8(NamedTuple):
    """8-bit values and the scales of every 32 of them in a row."""
    q: object       # [..., D] float8_e4m3fn
    scales: object  # [..., ceil(D / 32)] float8_e8m0fnu


class Norm(NamedTuple):
    """isc_rmsnorm's outputs; None for those not asked for."""
    y: object
    h: object
    mx8: object
    rstd: object


class Route(NamedTuple):
    """isc_route's outputs; offsets and order are None without lists."""
    ids: object      # [T, k] int32, -1 in an empty slot
    weights: object  # [T, k] float32
    offsets: object  # [E + 1] int32
    order: object    # [T * k] int32


class W4:
    """Packed 4-bit weights (isc_w4_pack_codes): `desc` and the device buffer;
    `stacked` if they are several matrices, for the experts of a route."""

    def __init__(self, desc, data, stacked):
        self.desc, self.data, self.stacked = desc, data, stacked
        self.E, self.N, self.K = desc.E, desc.N, desc.K


def declare(L):
    """The argument types of the C functions."""
    i32, i64, sz, vp, f32 = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_float
    dp, szp = ctypes.POINTER(W4Desc), ctypes.POINTER(sz)
    L.isc_rmsnorm.argtypes = [i32, i32, i32, vp, i64, vp, i64, vp, i32, f32, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp]
    L.isc_rmsnorm_bwd_workspace_size.argtypes = [i32, i32, szp]
    L.isc_rmsnorm_bwd.argtypes = [i32, i32, i32, vp, i64, vp, i64, vp, i32, vp, vp, i64, vp, i64, vp, vp, sz, vp]
    L.isc_route_workspace_size.argtypes = [i32, i32, szp]
    L.isc_route.argtypes = [i32, i32, i32, i32, vp, i64, vp, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp, sz, vp]
    L.isc_route_bwd.argtypes = [i32, i32, i32, i32, vp, vp, i64, vp, i32, i32, f32, vp, i64, vp]
    L.isc_w4_size.argtypes = [dp, szp]
    L.isc_w4_quantize.argtypes = [dp, vp, i32, i64, vp, vp, vp]
    L.isc_w4_pack_codes.argtypes = [dp, vp, vp, vp, vp]
    L.isc_w4_linear_workspace_size.argtypes = [dp, i32, i32, i32, szp]
    L.isc_w4_linear.argtypes = [dp, vp, i32, vp, i32, i64, vp, i64, i32, vp, vp, vp, vp, i32, i64, i32, vp, sz, vp]
    L.isc_w4_skip_workspace_size.argtypes = [dp, i32, i32, szp]
    L.isc_w4_skip.argtypes = [dp, vp, i32, vp, i32, i64, i32, vp, vp, vp, i32, i64, vp, sz, vp]


_state = None


class _State:
    """What every call needs, looked up once: the library, torch's types and
    its query for the current stream of a device."""

    def __init__(self):
        torch = _isc._torch()
        self.torch, self.lib = torch, _isc.lib()
        self.types = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
        self.f8, self.e8, self.f32, self.i32, self.u8 = (torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.float32,
                                                         torch.int32, torch.uint8)
        # the stream's handle itself where torch hands it out: a Stream object costs
        # 2.8 us, a fifth of a one-token call
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.stream_of = raw or (lambda device: torch.cuda.current_stream(device).cuda_stream)
        self.device = torch.cuda.current_device
        self.like = torch.empty_like


def _ready():
    global _state
    if _state is None:
        _state = _State()
    return _state


def _type(st, dtype, name):
    """The isc_type of a dtype."""
    code = st.types.get(dtype)
    if code is None:
        raise TypeError("%s must be float32, float16 or bfloat16, not %s" % (name, dtype))
    return code


def _stream(st, stream, device):
    return st.stream_of(device) if stream is None else _isc._stream(stream)


def _device(st, first, *others):
    """The index of the device that holds every tensor given; it is the current one."""
    index = first.get_device()
    if index < 0 or index != st.device():
        raise ValueError("tensors must be on the current CUDA/HIP device, not on %s" % first.device)
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError("tensors are on %s and %s" % (first.device, t.device))
    return index


def _rows(t, cols, name):
    """(tensor, leading dimension) of t as rows of `cols` values: t itself where its
    rows are evenly spaced and do not overlap, else a contiguous copy."""
    sizes = t.shape
    if not sizes or sizes[-1] != cols:
        raise ValueError("%s must have %d values in its last dimension, not %r" % (name, cols, tuple(sizes)))
    if t.is_contiguous():
        return t, cols
    strides = t.stride()
    if len(sizes) > 1 and (strides[-1] == 1 or cols == 1):
        ld, span = None, 1
        for n, s in zip(reversed(sizes[:-1]), reversed(strides[:-1])):
            if n == 1:
                continue
            if ld is None:
                ld = s
            elif s != ld * span:
                ld = 0
                break
            span *= n
        if ld is None:
            return t, cols
        if ld >= cols:
            return t, ld
    return t.contiguous(), cols


def _vector(t, n, name):
    if t.dim() != 1 or t.shape[0] != n:
        raise ValueError("%s must be [%d], not %r" % (name, n, tuple(t.shape)))
    return t if t.is_contiguous() else t.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _exact(t, dtype, shape, name):
    """A contiguous tensor of that type and shape."""
    if t.dtype != dtype or t.shape != shape:
        raise ValueError("%s must be %s %r, not %s %r" % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    return t if t.is_contiguous() else t.contiguous()


@functools.lru_cache(maxsize=4096)
def _size(query, *shape):
    """Bytes of workspace that a size query of the library gives for a shape."""
    n = ctypes.c_size_t()
    _isc._check(getattr(_isc.lib(), query)(*shape, n), query)
    return n.value


@functools.lru_cache(maxsize=4096)
def _w4_size(query, E, N, K, layout, *call):
    """The same for a call with packed weights."""
    return _size.__wrapped__(query, W4Desc(E, N, K, layout), *call)


def _on_stream(call):
    """call(st, ..., stream) with its temporaries allocated on the call's stream;
    st, the package's state, is not the caller's to give."""
    @functools.wraps(call)
    def run(*args, stream=None, **kw):
        st = _state or _ready()
        if stream is None:
            return call(st, *args, **kw)
        with _isc._on(stream):
            return call(st, *args, stream=stream, **kw)
    own = inspect.signature(call)
    run.__signature__ = own.replace(parameters=list(own.parameters.values())[1:])
    return run


def _new(st, like, dtype, *shape):
    """A contiguous tensor on like's device, by torch's quickest way: a one-token call
    spends more time on its outputs than on the GPU."""
    if len(shape) == 2:
        strides = (shape[1], 1)
    else:
        strides, n = [], 1
        for size in reversed(shape):
            strides.append(n)
            n *= size
        strides.reverse()
    return st.torch.empty_strided(shape, strides, dtype=dtype, device=like.device)


def _bytes(st, n, like):
    """A workspace of n bytes."""
    return st.torch.empty_strided((n,), (1,), dtype=st.u8, device=like.device)


@_on_stream
def isc_rmsnorm(st, x, weight, eps=1e-6, residual=None, y=True, mx8=False, rstd=False, stream=None):
    """h = x + residual, and its root-mean-square norm times `weight`, over the last dimension.

    x: [..., D] float32, float16 or bfloat16; residual: as x, or None; weight: [D]
    of any of those types.  Returns Norm(y, h, mx8, rstd): y in x's type (if y),
    h (with a residual), the norm in 8 bits with scales (if mx8), the reciprocal
    root mean squares for isc_rmsnorm_bwd (if rstd)."""
    if not (y or mx8 or rstd or residual is not None):
        raise ValueError("nothing is asked for")
    shape = x.shape
    D = shape[-1]
    code = _type(st, x.dtype, "x")
    device = _device(st, x, weight, residual)
    xr, ldx = _rows(x, D, "x")
    rp, ldr, h, hp, out, yp, form, qp, sp = None, D, None, None, None, None, None, None, None
    if residual is not None:
        if residual.dtype != x.dtype or residual.shape != shape:
            raise ValueError("residual must have x's shape and type")
        rr, ldr = _rows(residual, D, "residual")
        rp = rr.data_ptr()
        h = st.like(xr) if ldx == D else _new(st, x, x.dtype, *shape)
        hp = h.data_ptr()
    wr = _vector(weight, D, "weight")
    if y:
        out = st.like(xr) if ldx == D else _new(st, x, x.dtype, *shape)
        yp = out.data_ptr()
    groups = (D + 31) // 32
    if mx8:
        q = st.like(xr, dtype=st.f8) if ldx == D else _new(st, x, st.f8, *shape)
        scales = _new(st, x, st.e8, *shape[:-1], groups)
        form, qp, sp = Mx8(q, scales), q.data_ptr(), scales.data_ptr()
    rs = _new(st, x, st.f32, *shape[:-1]) if rstd else None
    status = st.lib.isc_rmsnorm(
        x.numel() // D if D else 0, D, code, xr.data_ptr(), ldx, rp, ldr, wr.data_ptr(),
        _type(st, wr.dtype, "weight"), eps, hp, D, yp, D, qp, D, sp, groups, _ptr(rs), _stream(st, stream, device))
    if status:
        _isc._check(status, "isc_rmsnorm")
    return Norm(out, h, form, rs)


@_on_stream
def isc_rmsnorm_bwd(st, dy, h, weight, rstd, dh=None, ws=None, stream=None):
    """The gradient of isc_rmsnorm: (dx, dweight).

    dy, h: [..., D] of one type, h as the forward pass gave it (x without a
    residual); rstd: [...] float32 from there; dh: the gradient that reaches h
    past the norm, or None.  dx (in h's type) is the gradient of x and of the
    residual alike; dweight is float32 [D]."""
    D = h.shape[-1]
    code = _type(st, h.dtype, "h")
    device = _device(st, h, dy, weight, rstd, dh, ws)
    for t, name in ((dy, "dy"), (dh, "dh")):
        if t is not None and (t.dtype != h.dtype or t.shape != h.shape):
            raise ValueError("%s must have h's shape and type" % name)
    T = h.numel() // D if D else 0
    rs = _exact(rstd, st.f32, h.shape[:-1], "rstd")
    hr, ldh = _rows(h, D, "h")
    yr, ldy = _rows(dy, D, "dy")
    gr, ldd = (None, D) if dh is None else _rows(dh, D, "dh")
    wr = _vector(weight, D, "weight")
    dx = st.like(hr) if ldh == D else _new(st, h, h.dtype, *h.shape)
    dw = _new(st, h, st.f32, D)
    if ws is None:
        ws = _bytes(st, _size("isc_rmsnorm_bwd_workspace_size", T, D), h)
    status = st.lib.isc_rmsnorm_bwd(
        T, D, code, yr.data_ptr(), ldy, hr.data_ptr(), ldh, wr.data_ptr(), _type(st, wr.dtype, "weight"),
        rs.data_ptr(), _ptr(gr), ldd, dx.data_ptr(), D, dw.data_ptr(), ws.data_ptr(), _isc._nbytes(ws),
        _stream(st, stream, device))
    if status:
        _isc._check(status, "isc_rmsnorm_bwd")
    return dx, dw


def _score(score):
    if score not in SCORES:
        raise ValueError("score must be one of %s, not %r" % (", ".join(SCORES), score))
    return SCORES[score]


@_on_stream
def isc_route(st, logits, k, bias=None, score="softmax", groups=1, keep_groups=None, renorm=True, scale=1.0, lists=True,
              ws=None, stream=None):
    """Each token's k experts, their weights, and the pairs by expert: Route(ids, weights, offsets, order).

    logits: [T, E] float32, float16 or bfloat16; bias: [E] float32, added to the
    scores for the choice only; groups, keep_groups: the choice is among the
    experts of the best keep_groups (default: all) of that many groups; renorm:
    weights divided by their sum; lists=False: no offsets and order."""
    which = _score(score)
    if logits.dim() != 2:
        raise ValueError("logits must be [T, E], not %r" % (tuple(logits.shape),))
    T, E = logits.shape
    code = _type(st, logits.dtype, "logits")
    device = _device(st, logits, bias, ws)
    lr, ld = _rows(logits, E, "logits")
    br = None if bias is None else _exact(bias, st.f32, (E,), "bias")
    k = int(k)
    if not 1 <= k <= E:
        raise ValueError("k must be 1 to %d, not %d" % (E, k))
    ids = _new(st, logits, st.i32, T, k)
    weights = st.like(ids, dtype=st.f32)
    offsets, order = (_new(st, logits, st.i32, E + 1), _new(st, logits, st.i32, T * k)) if lists else (None, None)
    if ws is None and lists and T > 16:
        n = _size("isc_route_workspace_size", T, E)
        ws = _bytes(st, n, logits) if n else None
    # an empty tensor has no address, and without tokens there is no order to write
    at = order.data_ptr() or offsets.data_ptr() if lists and not T else _ptr(order)
    status = st.lib.isc_route(
        T, E, k, code, lr.data_ptr(), ld, _ptr(br), which, groups, groups if keep_groups is None else keep_groups,
        bool(renorm), scale, ids.data_ptr(), weights.data_ptr(), _ptr(offsets), at, _ptr(ws),
        0 if ws is None else _isc._nbytes(ws), _stream(st, stream, device))
    if status:
        _isc._check(status, "isc_route")
    return Route(ids, weights, offsets, order)


@_on_stream
def isc_route_bwd(st, dweights, logits, ids, score="softmax", renorm=True, scale=1.0, stream=None):
    """The gradient of isc_route's weights to its logits, in their type.

    dweights: [T, k] float32; ids: [T, k] int32 as isc_route gave them; score,
    renorm, scale: as there."""
    which = _score(score)
    if logits.dim() != 2 or ids.dim() != 2:
        raise ValueError("logits must be [T, E] and ids [T, k]")
    T, E = logits.shape
    k = ids.shape[1]
    code = _type(st, logits.dtype, "logits")
    device = _device(st, logits, dweights, ids)
    lr, ld = _rows(logits, E, "logits")
    dr = _exact(dweights, st.f32, (T, k), "dweights")
    ir = _exact(ids, st.i32, (T, k), "ids")
    out = st.like(lr) if ld == E else _new(st, logits, logits.dtype, T, E)
    status = st.lib.isc_route_bwd(T, E, k, code, dr.data_ptr(), lr.data_ptr(), ld, ir.data_ptr(), which, bool(renorm),
                                  scale, out.data_ptr(), E, _stream(st, stream, device))
    if status:
        _isc._check(status, "isc_route_bwd")
    return out


@_on_stream
def isc_w4_quantize(st, w, stream=None):
    """(codes, scales) of 4-bit weights: w [N, K] or [E, N, K] float32, float16 or
    bfloat16; codes [..., N, ceil(K / 2)] uint8, scales [..., N, ceil(K / 32)] float8_e8m0fnu."""
    torch = st.torch
    if w.dim() not in (2, 3):
        raise ValueError("w must be [N, K] or [E, N, K], not %r" % (tuple(w.shape),))
    E = w.shape[0] if w.dim() == 3 else 1
    N, K = w.shape[-2:]
    device = _device(st, w)
    wr, ld = _rows(w, K, "w")
    codes = torch.empty((*w.shape[:-1], (K + 1) // 2), dtype=torch.uint8, device=w.device)
    scales = torch.empty((*w.shape[:-1], (K + 31) // 32), dtype=torch.float8_e8m0fnu, device=w.device)
    _isc._check(st.lib.isc_w4_quantize(W4Desc(E, N, K, 0), wr.data_ptr(), _type(st, w.dtype, "w"), ld,
                                       codes.data_ptr(), scales.data_ptr(), _stream(st, stream, device)),
                "isc_w4_quantize")
    return codes, scales


@_on_stream
def isc_w4_pack_codes(st, codes, scales, layout, K=None, stream=None):
    """The packed weights (a W4) of codes [N, K / 2] or [E, N, K / 2] and their scales.

    layout: "tiles" for isc_w4_linear, "rows" for isc_w4_skip; K: the number of
    inputs where it is odd (the last byte's high half is then ignored)."""
    torch = st.torch
    if layout not in LAYOUTS:
        raise ValueError("layout must be one of %s, not %r" % (", ".join(LAYOUTS), layout))
    if codes.dim() not in (2, 3) or codes.dtype != torch.uint8:
        raise ValueError("codes must be uint8 [N, K / 2] or [E, N, K / 2]")
    K = 2 * codes.shape[-1] if K is None else int(K)
    if (K + 1) // 2 != codes.shape[-1]:
        raise ValueError("codes have %d bytes a row, not those of %d inputs" % (codes.shape[-1], K))
    if scales.dtype not in (torch.float8_e8m0fnu, torch.uint8) or \
            tuple(scales.shape) != (*codes.shape[:-1], (K + 31) // 32):
        raise ValueError("scales must be float8_e8m0fnu or uint8 %r" % ((*codes.shape[:-1], (K + 31) // 32),))
    device = _device(st, codes, scales)
    E = codes.shape[0] if codes.dim() == 3 else 1
    desc = W4Desc(E, codes.shape[-2], K, LAYOUTS[layout])
    n = ctypes.c_size_t()
    _isc._check(st.lib.isc_w4_size(desc, n), "isc_w4_size")
    data = _bytes(st, n.value, codes)
    cr, sr = codes.contiguous(), scales.contiguous()
    _isc._check(st.lib.isc_w4_pack_codes(desc, cr.data_ptr(), sr.data_ptr(), data.data_ptr(),
                                         _stream(st, stream, device)), "isc_w4_pack_codes")
    return W4(desc, data, codes.dim() == 3)


def _routed(st, route, w4, T):
    """The slots per token and the route's tensors, checked."""
    if route is None:
        if w4.stacked:
            raise ValueError("weights of several matrices need a route")
        return 0, None, None, None, None
    if not w4.stacked:
        raise ValueError("a route needs weights of several matrices")
    ids, weights, offsets, order = route
    if ids.dim() != 2 or ids.shape[0] != T:
        raise ValueError("the route has %r slots, x %d tokens" % (tuple(ids.shape), T))
    slots = ids.shape[1]
    return slots, _exact(ids, st.i32, (T, slots), "ids"), weights, offsets, order


@_on_stream
def isc_w4_linear(st, x, w4, route=None, relu=False, dtype=None, ws=None, stream=None):
    """y = x w^T on 4-bit weights (layout "tiles"), with max(0, .) if relu.

    x: [..., K] float32, float16 or bfloat16, or an Mx8 (values, scales).
    Without a route: y is [..., N].  With one: x is [T, K], w4 holds the experts'
    matrices, and y is [T, k, N], slot j by the token's j-th expert (0 where it
    has none).  dtype: y's (default: x's, bfloat16 for an Mx8)."""
    K, N = w4.K, w4.N
    sp, lds, scales = None, 0, None
    if isinstance(x, tuple):
        x, scales = x
        if x.dtype != st.f8 or scales.dtype != st.e8:
            raise TypeError("an Mx8 is float8_e4m3fn values and float8_e8m0fnu scales")
        if scales.shape[:-1] != x.shape[:-1]:
            raise ValueError("scales are %r, for values %r" % (tuple(scales.shape), tuple(x.shape)))
        code = MX8
        scales, lds = _rows(scales, (K + 31) // 32, "scales")
        sp = scales.data_ptr()
    else:
        code = _type(st, x.dtype, "x")
    shape = x.shape
    xr, ldx = _rows(x, K, "x")
    T = x.numel() // K
    if route is not None and len(shape) != 2:
        raise ValueError("x must be [T, K] with a route")
    slots, ids, _, offsets, order = _routed(st, route, w4, T)
    device = _device(st, x, scales, w4.data, ids, offsets, order, ws)
    if slots:
        if offsets is None or order is None:
            raise ValueError("the route has no lists")
        offsets = _exact(offsets, st.i32, (w4.E + 1,), "offsets")
        order = _exact(order, st.i32, (T * slots,), "order")
    if dtype is None:
        dtype = st.torch.bfloat16 if code == MX8 else x.dtype
    if ws is None and not slots and 3 * T > COLUMNS[code]:
        n = _w4_size("isc_w4_linear_workspace_size", w4.E, N, K, LAYOUTS["tiles"], T, code, 0)
        ws = _bytes(st, n, x) if n else None
    y = _new(st, x, dtype, T, slots, N) if slots else _new(st, x, dtype, *shape[:-1], N)
    status = st.lib.isc_w4_linear(
        w4.desc, w4.data.data_ptr(), T, xr.data_ptr(), code, ldx, sp, lds, slots, _ptr(ids), _ptr(offsets),
        _ptr(order), y.data_ptr(), _type(st, dtype, "dtype"), N, bool(relu), _ptr(ws),
        0 if ws is None else _isc._nbytes(ws), _stream(st, stream, device))
    if status:
        _isc._check(status, "isc_w4_linear")
    return y


@_on_stream
def isc_w4_skip(st, x, w4, route=None, dtype=None, ws=None, stream=None):
    """y = x w^T on 4-bit weights (layout "rows") for a rectified x: zeros are skipped and
    their weights not read.

    Without a route: x is [..., K], y [..., N].  With one: x is [T, k, K]
    (isc_w4_linear's output), and y [T, N] the sum over a token's experts under
    the route's weights.  dtype: y's (default: x's)."""
    K, N = w4.K, w4.N
    shape = x.shape
    code = _type(st, x.dtype, "x")
    xr, ldx = _rows(x, K, "x")
    if route is not None and len(shape) != 3:
        raise ValueError("x must be [T, k, K] with a route")
    T = shape[0] if route is not None else x.numel() // K
    slots, ids, weights, _, _ = _routed(st, route, w4, T)
    device = _device(st, x, w4.data, ids, weights, ws)
    if slots:
        if shape[1] != slots:
            raise ValueError("x has %d slots, the route %d" % (shape[1], slots))
        weights = _exact(weights, st.f32, (T, slots), "weights")
    if ws is None:
        n = _w4_size("isc_w4_skip_workspace_size", w4.E, N, K, LAYOUTS["rows"], T, slots)
        if n:
            ws = _bytes(st, n, x)
    dtype = x.dtype if dtype is None else dtype
    y = _new(st, x, dtype, T, N) if slots else _new(st, x, dtype, *shape[:-1], N)
    status = st.lib.isc_w4_skip(
        w4.desc, w4.data.data_ptr(), T, xr.data_ptr(), code, ldx, slots, _ptr(ids), _ptr(weights), y.data_ptr(),
        _type(st, dtype, "dtype"), N, _ptr(ws), 0 if ws is None else _isc._nbytes(ws),
        _stream(st, stream, device))
    if status:
        _isc._check(status, "isc_w4_skip")
    return y
