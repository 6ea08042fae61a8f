"""The feed-forward operators on the GPU against their 64-bit forms.

Tolerances, from the arithmetic (u: half a unit in the last place of the
output's type relative to the value, 2^-24, 2^-11, 2^-8; e = 2^-24):
  norm        a sum of D squares, at most 64 of them in a row and the rest by a
              tree: under 100 e; the square root, the quotient and two products
              a few more: 128 e |y| + u |y|.  In 8 bits: half a step of the
              value's binade, 2^-4 of it or 2^-10 of the scale.
  gradients   the same bound on each term's size, times the longest run of
              additions
  products    (K + 64) e times the sum of |w x|: no order of fp32 additions errs
              more, with as much again for the matrix cores' aligned products;
              plus u |y|
"""
import ctypes
import sys

import numpy as np
import pytest

from oracle import ffn

pytestmark = pytest.mark.gpu

E24 = 2.0 ** -24
U = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TYPES = ["float32", "float16", "bfloat16"]
TINY = 2.0 ** -24  # half the smallest fp16 number, the coarsest of the types near zero


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available()
    return t


@pytest.fixture(scope="module")
def isc(torch):
    import paper_1704_07724_amd as m
    m.lib()
    return m


def note(*parts):
    print("[case]", *parts, flush=True)
    sys.stdout.flush()


def host(t):
    """A tensor's values in 64 bits, or its bytes for the 8-bit types."""
    import torch
    if t.dtype in (torch.float8_e4m3fn, torch.float8_e8m0fnu):
        return t.view(torch.uint8).cpu().numpy()
    return t.cpu().double().numpy() if t.dtype.is_floating_point else t.cpu().numpy()


def dev(torch, a, dtype="float32"):
    return torch.from_numpy(np.ascontiguousarray(a)).to(getattr(torch, dtype)).cuda()


def strided(t, extra, shift=0):
    """t's values in rows `extra` values further apart, starting `shift` values in."""
    import torch
    buf = torch.full((t.shape[0] * (t.shape[1] + extra) + shift,), 7, dtype=torch.float32).to(t.dtype).to(t.device)
    v = buf[shift:].view(t.shape[0], t.shape[1] + extra)[:, : t.shape[1]]
    v.copy_(t)
    return v


def close(got, want, size, dtype, what):
    """|got - want| <= size + u |want|, NaN and infinities in the same places."""
    got, want = np.broadcast_arrays(got, want)
    same = (np.isnan(got) & np.isnan(want)) | (got == want)
    with np.errstate(all="ignore"):
        ok = same | (np.abs(got - want) <= size + U[dtype] * np.abs(want) + TINY * (dtype == "float16"))
    if not ok.all():
        i = np.argwhere(~ok)[0]
        raise AssertionError("%s: %d of %d off; first at %s: %r, not %r" % (what, (~ok).sum(), ok.size, i, got[tuple(i)],
                                                                          want[tuple(i)]))


# ------------------------------------------------------------------- norm --

NORMS = [(1, 1), (3, 2), (2, 7), (5, 31), (4, 32), (1, 33), (7, 64), (3, 511), (2, 512), (2, 513), (66, 1000), (1, 4096),
         (3, 8191), (2, 8200), (2, 16384), (1, 20000), (1, 65536)]


def check_mx8(q, scales, y, size):
    """8-bit rows against the 64-bit norm: their scales, and values within half a step."""
    e = ffn.scale_exponents(y, 448.0) + 127
    lo = ffn.scale_exponents(y * (1 - 1e-5), 448.0) + 127  # a largest value that rounding moves past a power of two
    hi = ffn.scale_exponents(y * (1 + 1e-5), 448.0) + 127
    assert ((scales >= np.minimum(lo, e)) & (scales <= np.maximum(hi, e))).all(), "group scales"
    s = np.repeat(ffn.scale_values(scales), 32, axis=-1)[..., : y.shape[-1]]
    v = ffn.mx8_values(q, scales)
    ok = np.abs(v - y) <= size + np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * s)
    assert (ok | np.isnan(s)).all(), "8-bit values"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D", NORMS)
def test_norm(torch, isc, T, D, dtype):
    note("norm", T, D, dtype)
    r = np.random.default_rng(T * 1000 + D)
    x, res = dev(torch, r.standard_normal((T, D)), dtype), dev(torch, r.standard_normal((T, D)) * 3, dtype)
    wtype = dtype if D % 2 else "float32"
    w = dev(torch, 1 + 0.2 * r.standard_normal(D), wtype)
    n = isc.isc_rmsnorm(x, w, eps=1e-5, residual=res, mx8=True, rstd=True)
    h, rstd, y = ffn.rmsnorm(host(x), host(w), 1e-5, host(res))
    close(host(n.h), h, E24 * np.abs(h), dtype, "h")
    close(host(n.rstd), rstd, 128 * E24 * rstd, "float32", "rstd")
    close(host(n.y), y, 128 * E24 * np.abs(y), dtype, "y")
    check_mx8(host(n.mx8.q), host(n.mx8.scales), y, 128 * E24 * np.abs(y))
    # each output alone, and without a residual
    only = isc.isc_rmsnorm(x, w, eps=1e-5)
    assert only.h is None and only.mx8 is None and only.rstd is None
    close(host(only.y), ffn.rmsnorm(host(x), host(w), 1e-5)[2], 128 * E24 * np.abs(y) * 4 + 1e-6, dtype, "y alone")
    again = isc.isc_rmsnorm(x, w, eps=1e-5, residual=res, y=False, mx8=True)
    assert np.array_equal(host(again.mx8.q), host(n.mx8.q)) and again.y is None


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("extra,shift", [(8, 0), (5, 0), (3, 1), (0, 1)])
@pytest.mark.parametrize("D", [40, 1000])
def test_norm_strides(torch, isc, D, extra, shift, dtype):
    """Rows further apart, and rows that start off a 16-byte boundary, give the same values."""
    note("norm strides", D, extra, shift, dtype)
    r = np.random.default_rng(D + extra)
    x, res, dy = (dev(torch, r.standard_normal((6, D)), dtype) for _ in range(3))
    w = dev(torch, r.standard_normal(D), dtype)
    a = isc.isc_rmsnorm(x, w, residual=res, mx8=True, rstd=True)
    xs, rs, ds = strided(x, extra, shift), strided(res, extra, shift), strided(dy, extra, shift)
    b = isc.isc_rmsnorm(xs, w, residual=rs, mx8=True, rstd=True)
    for u, v in ((a.y, b.y), (a.h, b.h), (a.mx8.q, b.mx8.q), (a.mx8.scales, b.mx8.scales), (a.rstd, b.rstd)):
        assert np.array_equal(host(u), host(v))
    g = isc.isc_rmsnorm_bwd(dy, a.h, w, a.rstd, dh=res)
    s = isc.isc_rmsnorm_bwd(ds, strided(a.h, extra, shift), w, a.rstd, dh=rs)
    assert all(np.array_equal(host(u), host(v)) for u, v in zip(g, s))
    # a broadcast row, a transposed batch, leading dimensions
    c = isc.isc_rmsnorm(x[:1].expand(6, D), w, residual=res)
    close(host(c.y), ffn.rmsnorm(np.repeat(host(x)[:1], 6, 0), host(w), 1e-6, host(res))[2],
          128 * E24 * 64, dtype, "broadcast x")
    t = isc.isc_rmsnorm(x.view(2, 3, D).transpose(0, 1), w)
    assert t.y.shape == (3, 2, D)
    assert np.array_equal(host(t.y), host(isc.isc_rmsnorm(x.view(2, 3, D).transpose(0, 1).contiguous(), w).y))


def test_norm_values(torch, isc):
    """Rows of zeros, of the smallest and of large numbers, with infinities and NaN: each row by itself."""
    note("norm values")
    D = 96
    x = np.random.default_rng(3).standard_normal((7, D)).astype(np.float32)
    x[0] = 0
    x[1] *= 1e-30
    x[2] *= 1e15
    x[3, 5] = np.inf
    x[4, 40] = np.nan
    x[5, 32:64] = 0
    w = np.ones(D, np.float32)
    n = isc.isc_rmsnorm(dev(torch, x), dev(torch, w), mx8=True, rstd=True)
    y, q, s = host(n.y), host(n.mx8.q), host(n.mx8.scales)
    rows = [0, 1, 2, 5, 6]
    want = ffn.rmsnorm(x[rows], w, 1e-6)[2]
    close(y[rows], want, 128 * E24 * np.abs(want), "float32", "y")
    assert (y[0] == 0).all() and (q[0] & 127 == 0).all() and (s[0] == 0).all()
    assert (s[5, 1] == 0) and (q[5, 32:64] & 127 == 0).all()
    assert np.isnan(y[3, 5]) and np.isnan(y[4]).all()
    assert s[3, 0] == 255 and (q[3, :32] & 127 == 127).all()  # the infinity's group
    assert (s[4] == 255).all()


@pytest.mark.parametrize("D", [40, 1001, 40000])
def test_norm_small_means(torch, isc, D):
    """Mean squares that fp32 holds below its smallest normal number, without an eps to hide them: down to
    2^-140 they have 9 bits and more, so the root errs by 2^-11 of itself at most."""
    note("norm small means", D)
    r = np.random.default_rng(D)
    powers = np.array([-60, -62, -63, -64, -66, -68, -70])
    h = np.sign(r.standard_normal((len(powers), D))) * 2.0 ** powers[:, None]
    w = 1 + 0.2 * r.standard_normal(D)
    n = isc.isc_rmsnorm(dev(torch, h), dev(torch, w), eps=0.0, rstd=True)
    # each square is exact; a sum's terms below 2^-126 are, too: they are multiples of 2^-140
    want = 2.0 ** -powers.astype(np.float64)
    assert (np.abs(host(n.rstd) - want) <= 2.0 ** -11 * want).all()
    y = h * want[:, None] * host(dev(torch, w))
    assert (np.abs(host(n.y) - y) <= 2.0 ** -11 * np.abs(y) + 2.0 ** -20).all()


def test_norm_no_rows(torch, isc):
    note("norm no rows")
    x, w = torch.empty((0, 64), device="cuda"), torch.ones(64, device="cuda")
    n = isc.isc_rmsnorm(x, w, residual=x, mx8=True, rstd=True)
    assert n.y.shape == (0, 64) and n.mx8.scales.shape == (0, 2) and n.rstd.shape == (0,)
    dx, dw = isc.isc_rmsnorm_bwd(x, x, w, n.rstd)
    assert dx.shape == (0, 64) and (host(dw) == 0).all()


@pytest.mark.parametrize("D,T", [(3, 2 ** 26 + 7), (24, 2 ** 26 + 1)])
def test_norm_more_rows_than_a_launch_takes(torch, isc, D, T):
    """The rows of the last launch and those on either side of its start, each output, as in a small call."""
    note("norm many rows", D, T)
    g = torch.Generator(device="cuda").manual_seed(D)
    x = torch.randn((T, D), generator=g, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(D, generator=g, device="cuda").bfloat16()
    got = isc.isc_rmsnorm(x, w, residual=x, mx8=True, rstd=True)
    cut = (2 ** 32 - 1) // 64
    for rows in (slice(0, 4), slice(cut - 4, cut + 4), slice(T - 4, T)):
        small = isc.isc_rmsnorm(x[rows], w, residual=x[rows], mx8=True, rstd=True)
        for a, b in ((got.y, small.y), (got.h, small.h), (got.mx8.q, small.mx8.q), (got.mx8.scales, small.mx8.scales),
                     (got.rstd, small.rstd)):
            assert np.array_equal(host(a[rows]), host(b)), rows
    # and no row in between was left out: every mean is that of its row
    step = 1 << 22
    for t in range(0, T, step):
        h = x[t:t + step].float() * 2
        want = torch.rsqrt((h * h).mean(-1) + 1e-6)
        assert ((got.rstd[t:t + step] - want).abs() <= 256 * E24 * want).all(), t


@pytest.mark.parametrize("D", [64, 1000, 16384])
def test_norm_bwd_no_rows_no_weight(torch, isc, D):
    """A call without rows needs none of their tensors, the weight among them: dw is 0."""
    note("norm bwd no rows, no weight", D)
    n = ctypes.c_size_t()
    assert isc.lib().isc_rmsnorm_bwd_workspace_size(0, D, n) == 0
    ws = torch.full((n.value,), 255, dtype=torch.uint8, device="cuda")
    dw = torch.full((D,), float("nan"), device="cuda")
    assert isc.lib().isc_rmsnorm_bwd(0, D, 2, None, D, None, D, None, 2, None, None, D, None, D, dw.data_ptr(),
                                     ws.data_ptr(), n.value, isc._stream(None)) == 0
    assert (host(dw) == 0).all()


def test_norm_in_place(torch, isc):
    """h written over the residual, and dx over dy, through the C entry points."""
    note("norm in place")
    r = np.random.default_rng(8)
    T, D = 5, 264
    x, res = dev(torch, r.standard_normal((T, D)), "bfloat16"), dev(torch, r.standard_normal((T, D)), "bfloat16")
    w = torch.ones(D, device="cuda", dtype=torch.bfloat16)
    want = isc.isc_rmsnorm(x, w, residual=res, rstd=True)
    run, buf, y, rstd = res.clone(), x.clone(), torch.empty_like(x), torch.empty(T, device="cuda")
    st = isc.lib().isc_rmsnorm(T, D, 2, buf.data_ptr(), D, run.data_ptr(), D, w.data_ptr(), 2, 1e-6, run.data_ptr(), D,
                               buf.data_ptr(), D, None, 0, None, 0, rstd.data_ptr(), isc._stream(None))
    assert st == 0
    assert torch.equal(run, want.h) and torch.equal(buf, want.y) and torch.equal(rstd, want.rstd)
    dx, dw = isc.isc_rmsnorm_bwd(y.copy_(res), want.h, w, rstd)
    n = ctypes.c_size_t()
    assert isc.lib().isc_rmsnorm_bwd_workspace_size(T, D, n) == 0
    ws, dw2 = torch.empty(n.value, dtype=torch.uint8, device="cuda"), torch.empty(D, device="cuda")
    st = isc.lib().isc_rmsnorm_bwd(T, D, 2, y.data_ptr(), D, want.h.data_ptr(), D, w.data_ptr(), 2, rstd.data_ptr(), None, 0,
                                   y.data_ptr(), D, dw2.data_ptr(), ws.data_ptr(), n.value, isc._stream(None))
    assert st == 0 and torch.equal(y, dx) and torch.equal(dw2, dw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [9, 10, 11, 12, 13, 14, 15, 17, 257, 511, 513, 1001, 2046, 4099, 8191, 8195])
def test_norm_uneven_widths(torch, isc, D, dtype):
    """Rows that end inside eight values, between NaNs: nothing of the row before, the row after or the
    values moved aside comes in, in both directions and in place."""
    note("norm uneven widths", D, dtype)
    r = np.random.default_rng(D)
    T = 5

    def held(scale):
        t = torch.full((T, D + 11), float("nan"), dtype=getattr(torch, dtype), device="cuda")
        t[:, 5:D + 5] = dev(torch, r.standard_normal((T, D)) * scale, dtype)
        return t[:, 5:D + 5]
    x, res, dy, dh = held(1), held(3), held(1), held(1)
    w = dev(torch, 1 + 0.2 * r.standard_normal(D), dtype)
    n = isc.isc_rmsnorm(x, w, eps=1e-5, residual=res, mx8=True, rstd=True)
    h, rstd, y = ffn.rmsnorm(host(x), host(w), 1e-5, host(res))
    close(host(n.h), h, E24 * np.abs(h), dtype, "h")
    close(host(n.rstd), rstd, 128 * E24 * rstd, "float32", "rstd")
    close(host(n.y), y, 128 * E24 * np.abs(y), dtype, "y")
    check_mx8(host(n.mx8.q), host(n.mx8.scales), y, 128 * E24 * np.abs(y))
    plain = [t.contiguous() for t in (x, res, dy, dh)]
    same = isc.isc_rmsnorm(plain[0], w, eps=1e-5, residual=plain[1], rstd=True)
    assert torch.equal(same.h, n.h) and torch.equal(same.y, n.y) and torch.equal(same.rstd, n.rstd)
    dx, dw = isc.isc_rmsnorm_bwd(dy, n.h, w, n.rstd, dh=dh)
    g, n1 = host(dy) * host(w), host(n.h) * host(n.rstd)[:, None]
    want = host(n.rstd)[:, None] * (g - n1 * (g * n1).mean(1, keepdims=True)) + host(dh)
    size = host(n.rstd)[:, None] * (np.abs(g) + np.abs(n1) * np.abs(g * n1).mean(1, keepdims=True)) + np.abs(host(dh))
    close(host(dx), want, 128 * E24 * size, dtype, "dx")
    close(host(dw), (host(dy) * n1).sum(0), 64 * E24 * np.abs(host(dy) * n1).sum(0), "float32", "dw")
    # dx over dy, h over x
    code = {"float32": 0, "float16": 1, "bfloat16": 2}[dtype]
    n_ws = ctypes.c_size_t()
    assert isc.lib().isc_rmsnorm_bwd_workspace_size(T, D, n_ws) == 0
    ws, dw2 = torch.empty(n_ws.value, dtype=torch.uint8, device="cuda"), torch.empty(D, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert isc.lib().isc_rmsnorm_bwd(T, D, code, plain[2].data_ptr(), D, n.h.data_ptr(), D, w.data_ptr(), code,
                                     n.rstd.data_ptr(), plain[3].data_ptr(), D, plain[2].data_ptr(), D, dw2.data_ptr(),
                                     ws.data_ptr(), n_ws.value, stream) == 0
    assert torch.equal(plain[2], dx) and torch.equal(dw2, dw)
    assert isc.lib().isc_rmsnorm(T, D, code, plain[0].data_ptr(), D, plain[1].data_ptr(), D, w.data_ptr(), code, 1e-5,
                                 plain[0].data_ptr(), D, None, D, None, D, None, (D + 31) // 32, None, stream) == 0
    assert torch.equal(plain[0], n.h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,D", [(1, 1), (2, 7), (3, 33), (65, 64), (700, 100), (5, 1000), (1, 4096), (9, 8200), (2, 16384),
                                 (2100, 520)])
def test_norm_bwd(torch, isc, T, D, dtype):
    note("norm bwd", T, D, dtype)
    r = np.random.default_rng(T + D)
    h, dy, dh = (dev(torch, r.standard_normal((T, D)), dtype) for _ in range(3))
    w = dev(torch, 1 + 0.2 * r.standard_normal(D), "float32" if D % 2 else dtype)
    rstd = isc.isc_rmsnorm(h, w, y=False, rstd=True).rstd
    for extra in (None, dh):
        dx, dw = isc.isc_rmsnorm_bwd(dy, h, w, rstd, dh=extra)
        rs = host(rstd)[:, None]
        n, g = host(h) * rs, host(dy) * host(w)
        want, wdw = ffn.rmsnorm_bwd(host(dy), host(h), host(w), host(rstd), None if extra is None else host(extra))
        size = 128 * E24 * rs * (np.abs(g) + np.abs(n) * np.abs(g * n).mean(-1, keepdims=True)) + 2 * E24 * np.abs(want)
        close(host(dx), want, size, dtype, "dx")
        close(host(dw), wdw, (T + 64) * E24 * np.abs(host(dy) * n).sum(0), "float32", "dw")
    assert all(torch.equal(a, b) for a, b in zip((dx, dw), isc.isc_rmsnorm_bwd(dy, h, w, rstd, dh=dh)))


def test_norm_bwd_against_differences(torch, isc):
    """The gradient along a direction against differences of the forward kernel: with a
    step of 2^-7 the third derivative leaves some 1e-4 of the value and fp32 sums of
    2000 terms some 1e-3 of their size over the step."""
    note("norm bwd differences")
    r = np.random.default_rng(12)
    T, D = 4, 500
    h, dy, v = (r.standard_normal((T, D)) for _ in range(3))
    w = 1 + 0.2 * r.standard_normal(D)
    hd, wd, dyd = dev(torch, h), dev(torch, w), dev(torch, dy)
    dx, dw = isc.isc_rmsnorm_bwd(dyd, hd, wd, isc.isc_rmsnorm(hd, wd, rstd=True).rstd)
    step = 2.0 ** -7

    def loss(hh, ww):
        return (host(isc.isc_rmsnorm(dev(torch, hh), dev(torch, ww)).y) * dy).sum()

    along = (loss(h + step * v, w) - loss(h - step * v, w)) / (2 * step)
    assert abs(along - (host(dx) * v).sum()) <= 1e-3 * np.abs(host(dx) * v).sum()
    u = r.standard_normal(D)
    along = (loss(h, w + step * u) - loss(h, w - step * u)) / (2 * step)
    assert abs(along - (host(dw) * u).sum()) <= 1e-3 * np.abs(host(dw) * u).sum()


# ------------------------------------------------------------------ route --

def apart(logits, bias, score, k):
    """Moves logits on until no two keys of a token are nearer than 1e-5 of their
    size unless they are equal: an index is then the same in 32 and 64 bits."""
    r = np.random.default_rng(99)
    for t in range(len(logits)):
        for _ in range(50):
            s, there = ffn.scores(logits[t], score)
            key = np.sort((s if bias is None else s + bias)[there])
            d = np.diff(key)
            if not ((d > 0) & (d < 1e-5 * np.maximum(np.abs(key[1:]), 1e-6))).any():
                break
            live = np.isfinite(logits[t])
            logits[t, live] = (r.standard_normal(live.sum()) * 1.5).astype(np.float16)
    return logits


def check_route(got, want, E):
    ids, weights, offsets, order = want
    assert np.array_equal(host(got.ids), ids), "ids"
    # exp to 2 units, a sum of up to 1024 by a tree of at most 24 additions, two quotients
    close(host(got.weights), weights, 64 * E24 * np.abs(weights), "float32", "weights")
    if got.offsets is not None:
        assert np.array_equal(host(got.offsets), offsets), "offsets"
        assert np.array_equal(host(got.order), order), "order"


ROUTES = [
    # T, E, k, score, bias, groups, keep, renorm
    (1, 1, 1, "softmax", False, 1, 1, True),
    (3, 2, 2, "sigmoid", True, 1, 1, True),
    (5, 7, 3, "softmax", False, 1, 1, False),
    (63, 60, 4, "sigmoid", False, 1, 1, True),
    (64, 64, 8, "softmax", True, 1, 1, True),
    (65, 65, 1, "softmax", False, 1, 1, True),
    (200, 128, 8, "softmax", False, 1, 1, True),
    (16, 256, 8, "sigmoid", True, 8, 4, True),
    (130, 60, 5, "sigmoid", True, 4, 2, False),
    (70, 12, 4, "softmax", True, 6, 2, True),
    (10, 64, 64, "softmax", False, 1, 1, True),
    (9, 64, 6, "sigmoid", True, 64, 10, True),
    (7, 1000, 10, "softmax", True, 1, 1, True),
    (66, 1024, 16, "sigmoid", True, 16, 3, True),
    (300, 513, 6, "softmax", False, 27, 9, True),
]


@pytest.mark.parametrize("case", ROUTES, ids=lambda c: "-".join(map(str, c)))
def test_route(torch, isc, case):
    T, E, k, score, with_bias, groups, keep, renorm = case
    note("route", case)
    r = np.random.default_rng(T * 7 + E)
    bias = (r.integers(-60, 61, E) * 0.001).astype(np.float32) if with_bias else None
    # values that fp16 and bfloat16 hold, so that every type sees the same logits
    logits = np.round(r.standard_normal((T, E)) * 1.5, 1)
    logits = dev(torch, logits, "bfloat16").float().cpu().numpy()
    logits = apart(logits, None if bias is None else bias.astype(np.float64), score, k)
    logits[T // 2, : E // 2] = -np.inf  # half of a token's experts gone
    if T > 3:
        logits[1] = -np.inf                       # all of them
        logits[2] = -np.inf
        logits[2, E - 1] = 0.5                    # all but one
        logits[3] = np.finfo(np.float32).min      # the type's lowest value everywhere: it still counts
    want = ffn.route(logits, k, bias, score, groups, keep, renorm, 2.5)
    bd = None if bias is None else dev(torch, bias)
    x = dev(torch, logits)
    got = isc.isc_route(x, k, bias=bd, score=score, groups=groups, keep_groups=keep, renorm=renorm, scale=2.5)
    check_route(got, want, E)
    again = isc.isc_route(strided(x, 3), k, bias=bd, score=score, groups=groups, keep_groups=keep, renorm=renorm,
                          scale=2.5, lists=False)
    assert torch.equal(again.ids, got.ids) and torch.equal(again.weights, got.weights) and again.order is None


@pytest.mark.parametrize("E,k,groups", [(64, 6, 1), (64, 20, 1), (100, 8, 20), (128, 8, 1), (256, 8, 8), (400, 8, 1), (603, 5, 9)])
@pytest.mark.parametrize("T", [17, 64, 65, 700, 4097, 8192, 8205])
def test_route_workgroups(torch, isc, T, E, k, groups):
    """Many tokens: each as in a small call, and the lists of all of them."""
    note("route workgroups", T, E, k, groups)
    r = np.random.default_rng(T + E)
    x = dev(torch, r.standard_normal((T, E)), "bfloat16")
    x[T // 3] = float("-inf")
    x[T // 2, 3:] = float("-inf")
    keep = max(1, groups // 2)
    got = isc.isc_route(x, k, score="sigmoid", groups=groups, keep_groups=keep)
    ids, weights_ = host(got.ids), host(got.weights)
    for t in sorted({0, 16 * (T // 32), max(0, T - 16)}):
        small = isc.isc_route(x[t:t + 16], k, score="sigmoid", groups=groups, keep_groups=keep)
        assert np.array_equal(ids[t:t + 16], host(small.ids))
        # k weights of fp32, in another order of summing
        assert np.abs(weights_[t:t + 16] - host(small.weights)).max() <= (k + 4) * E24
    flat = ids.reshape(-1)
    order = np.argsort(np.where(flat < 0, E, flat), kind="stable")
    n = int((flat >= 0).sum())
    assert host(got.offsets).tolist() == np.concatenate([[0], np.cumsum(np.bincount(flat[flat >= 0], minlength=E))]).tolist()
    assert np.array_equal(host(got.order)[:n], order[:n]) and (host(got.order)[n:] == -1).all()


MANY = [
    # T, E, k, score, bias, groups, keep, renorm: tokens enough for four a wavefront, up to 64, 128 and 256 experts
    (17, 65, 3, "softmax", True, 1, 1, True),
    (64, 128, 8, "sigmoid", False, 1, 1, False),
    (50, 100, 16, "softmax", False, 10, 3, True),
    (61, 40, 4, "softmax", True, 4, 2, True),
    (4097, 128, 8, "softmax", False, 1, 1, True),
    (4099, 256, 8, "sigmoid", True, 8, 4, True),
    (4100, 129, 5, "softmax", True, 1, 1, False),
    (4101, 200, 16, "softmax", True, 10, 4, True),
    (4097, 250, 6, "sigmoid", False, 1, 1, True),
    (4098, 64, 2, "sigmoid", True, 16, 5, True),
    (8195, 90, 4, "softmax", False, 1, 1, True),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", MANY, ids=lambda c: "-".join(map(str, c)))
def test_route_many_tokens(torch, isc, case, dtype):
    """Every token of a call that routes four a wavefront, masked ones among them, in every type."""
    T, E, k, score, with_bias, groups, keep, renorm = case
    note("route many tokens", case, dtype)
    r = np.random.default_rng(T + 3 * E)
    bias = (r.integers(-60, 61, E) * 0.001).astype(np.float32) if with_bias else None
    # values that every type holds
    logits = host(dev(torch, np.round(r.standard_normal((T, E)) * 1.5, 1), "bfloat16"))
    logits[r.random((T, E)) < 0.1] = -np.inf
    # tokens whose choice hangs on fp32's rounding of two keys, or of two groups' sums, lose all their experts
    key = np.stack([ffn.scores(l, score)[0] for l in logits]) + (0.0 if bias is None else bias.astype(np.float64))
    key[logits == -np.inf] = -9.0
    best = np.sort(key.reshape(T, groups, -1), -1)[..., -2:].sum(-1)
    for v in [key] + [best] * (groups > 1):
        d = np.diff(np.sort(v, -1), axis=-1)
        logits[((d > 0) & (d < 1e-6)).any(-1)] = -np.inf
    assert (logits > -np.inf).any(1).mean() > 0.5
    x = dev(torch, logits, dtype)
    want = ffn.route(host(x), k, bias, score, groups, keep, renorm, 2.5)
    got = isc.isc_route(x, k, bias=None if bias is None else dev(torch, bias), score=score, groups=groups, keep_groups=keep,
                        renorm=renorm, scale=2.5)
    check_route(got, want, E)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_route_types_and_ties(torch, isc, dtype):
    """Coarse logits: many exact ties, each to the lowest index."""
    note("route ties", dtype)
    r = np.random.default_rng(4)
    logits = dev(torch, np.round(r.standard_normal((150, 96)) * 2) / 2, dtype)
    for score, groups, keep in (("softmax", 1, 1), ("sigmoid", 8, 3)):
        got = isc.isc_route(logits, 7, score=score, groups=groups, keep_groups=keep)
        check_route(got, ffn.route(host(logits), 7, None, score, groups, keep), 96)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [9, 40, 5000])
@pytest.mark.parametrize("E,k,groups,keep,step,bias", [(64, 12, 1, 1, 16.0, False), (200, 30, 1, 1, 16.0, False),
                                                       (700, 12, 1, 1, 16.0, False), (24, 24, 1, 1, 4.0, True),
                                                       (24, 12, 4, 2, 4.0, True), (24, 12, 4, 2, 4.0, False)])
def test_route_logits_far_apart(torch, isc, E, k, groups, keep, step, bias, T, dtype):
    """Experts whose softmax scores are hundreds of powers of e apart, or below fp32's smallest normal number beside a
    bias of 0: each still has its place.  Weights err by a few of the smallest fp32 numbers where they are that small."""
    note("route far apart", E, k, groups, keep, step, bias, T, dtype)
    r = np.random.default_rng(E + T)
    l = np.stack([np.minimum(r.permutation(E), 255) * -step for _ in range(T)])  # (as bfloat16 holds them)
    x = dev(torch, l, dtype)
    assert np.array_equal(host(x), l)
    got = isc.isc_route(x, k, bias=torch.zeros(E, device="cuda") if bias else None, groups=groups, keep_groups=keep)
    if T <= 40:
        want = ffn.route(l, k, np.zeros(E) if bias else None, groups=groups, keep=keep)
        for a, b in zip((got.ids, got.offsets, got.order), (want[0], *want[2:])):
            assert np.array_equal(host(a), b)
        assert (np.abs(host(got.weights) - want[1]) <= 64 * E24 * want[1] + 2.0 ** -147).all()
    elif groups == 1:
        assert np.array_equal(host(got.ids), np.argsort(-l, axis=1, kind="stable")[:, :k])
    small = isc.isc_route(x[:9], k, bias=torch.zeros(E, device="cuda") if bias else None, groups=groups, keep_groups=keep)
    assert torch.equal(small.ids, got.ids[:9])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [9, 5000])
def test_route_sigmoid_far_apart(torch, isc, T, dtype):
    """Confident experts, whose sigmoids are 1 in fp32, and faint ones, below its smallest normal number."""
    note("route sigmoid far apart", T, dtype)
    r, E, k = np.random.default_rng(T), 120, 60
    l = np.stack([r.permutation(E) - 90.0 for _ in range(T)])
    got = isc.isc_route(dev(torch, l, dtype), k, score="sigmoid", renorm=False)
    assert np.array_equal(host(got.ids), np.argsort(-l, axis=1, kind="stable")[:, :k])
    faint = isc.isc_route(dev(torch, l - 29.0, dtype), k, score="sigmoid", renorm=False)
    assert np.array_equal(host(faint.ids), host(got.ids))
    for g, shift in ((got, 0.0), (faint, 29.0)):
        want = 1 / (1 + np.exp(shift - np.take_along_axis(l, host(got.ids).astype(np.int64), 1)))
        assert (np.abs(host(g.weights) - want) <= 64 * E24 * want + 2.0 ** -147).all()


def test_route_values(torch, isc):
    """NaN and infinite logits, a bias that shuts an expert out, no tokens."""
    note("route values")
    inf, nan = np.inf, np.nan
    l = np.array([[0.0, nan, 1.0, -inf], [inf, 0.0, inf, 1.0], [nan] * 4, [-inf, -3e38, -3e38, -inf]], dtype=np.float32)
    for score in ("softmax", "sigmoid"):
        check_route(isc.isc_route(dev(torch, l), 3, score=score), ffn.route(l, 3, score=score), 4)
    bias = np.array([0.1, -inf, nan, 0.0], dtype=np.float32)
    l = np.zeros((1, 4), dtype=np.float32)
    got = isc.isc_route(dev(torch, l), 3, bias=dev(torch, bias))
    assert host(got.ids).tolist() == [[0, 3, -1]]
    got = isc.isc_route(torch.empty((0, 5), device="cuda"), 2)
    assert got.ids.shape == (0, 2) and host(got.offsets).tolist() == [0] * 6 and got.order.shape == (0,)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k,score,renorm", [(1, 1, 1, "sigmoid", False), (3, 7, 2, "softmax", True),
                                                (65, 64, 8, "sigmoid", True), (33, 128, 8, "softmax", False),
                                                (70, 300, 6, "softmax", True), (9, 1024, 64, "sigmoid", True)])
def test_route_bwd(torch, isc, T, E, k, score, renorm, dtype):
    note("route bwd", T, E, k, score, renorm, dtype)
    r = np.random.default_rng(T + E)
    logits = dev(torch, r.standard_normal((T, E)) * 1.5, dtype)
    if T > 3:
        logits[1, : E - 1] = float("-inf")
        logits[2] = float("-inf")
    dw = dev(torch, r.standard_normal((T, k)))
    ids = isc.isc_route(logits, k, score=score).ids
    got = isc.isc_route_bwd(dw, logits, ids, score=score, renorm=renorm, scale=1.5)
    l, i = host(logits), host(ids)
    want = ffn.route_bwd(host(dw), l, i, score, renorm, 1.5)
    # each term's size: the scores' gradients before they cancel
    size = np.zeros((T, E))
    for t in range(T):
        s, _ = ffn.scores(l[t], score)
        on = [(j, e) for j, e in enumerate(i[t]) if e >= 0]
        total = sum(s[e] for _, e in on) + 1e-20
        dot = sum(abs(host(dw)[t, j]) * s[e] for j, e in on)
        ds = np.zeros(E)
        for j, e in on:
            ds[e] = 1.5 * ((abs(host(dw)[t, j]) + dot / total) / total if renorm else abs(host(dw)[t, j]))
        size[t] = s * (ds + (ds * s).sum())
    close(host(got), want, 128 * E24 * size, dtype, "dlogits")
    s = isc.isc_route_bwd(dw, strided(logits, 5), ids, score=score, renorm=renorm, scale=1.5)
    assert np.array_equal(host(s), host(got))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k,renorm", [(1, 40, 40, False), (33, 60, 8, False), (33, 60, 8, True), (9, 300, 20, False)])
def test_route_bwd_confident(torch, isc, T, E, k, renorm, dtype):
    """Sigmoids near 1 and near 0: the gradient is to be right beside s (1 - s), not beside s."""
    note("route bwd confident", T, E, k, renorm, dtype)
    r = np.random.default_rng(T + E)
    l = host(dev(torch, r.choice([-1.0, 1.0], (T, E)) * r.uniform(8, 30, (T, E)), dtype))
    x, dw = dev(torch, l, dtype), dev(torch, r.standard_normal((T, k)))
    ids = isc.isc_route(x, k, score="sigmoid").ids
    got = host(isc.isc_route_bwd(dw, x, ids, score="sigmoid", renorm=renorm))
    s, c, d, i = 1 / (1 + np.exp(-l)), 1 / (1 + np.exp(l)), host(dw), host(ids).astype(np.int64)
    on = np.take_along_axis(s, i, 1)
    total = on.sum(1, keepdims=True) + 1e-20
    ds, size = np.zeros((T, E)), np.zeros((T, E))
    np.put_along_axis(ds, i, (d - (d * on).sum(1, keepdims=True) / total) / total if renorm else d, 1)
    np.put_along_axis(size, i, (np.abs(d) + (np.abs(d) * on).sum(1, keepdims=True) / total) / total if renorm else np.abs(d), 1)
    close(got, ds * s * c, 128 * E24 * size * s * c, dtype, "dlogits")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k,score,renorm,bias", [(33, 60, 8, "softmax", False, False), (33, 60, 8, "softmax", True, False),
                                                     (9, 300, 20, "softmax", False, True), (40, 128, 8, "softmax", True, True),
                                                     (5, 7, 2, "softmax", False, True), (33, 60, 8, "sigmoid", True, False),
                                                     (9, 1024, 64, "sigmoid", True, True), (6, 3, 1, "softmax", True, False)])
def test_route_bwd_dominant(torch, isc, T, E, k, score, renorm, bias, dtype):
    """One expert with nearly all of a sum, chosen first, later or not at all: its gradient is to be right beside the
    shares that the others have, since its own part of the sum goes out."""
    note("route bwd dominant", T, E, k, score, renorm, bias, dtype)
    r = np.random.default_rng(T + E)
    l = r.standard_normal((T, E)) - 12 * (score == "sigmoid")
    l[np.arange(T), r.integers(0, E, T)] += r.uniform(5, 25, T)
    x, dw = dev(torch, l, dtype), dev(torch, r.standard_normal((T, k)))
    ids = isc.isc_route(x, k, bias=dev(torch, r.standard_normal(E)) if bias else None, score=score).ids
    got = host(isc.isc_route_bwd(dw, x, ids, score=score, renorm=renorm))
    l, i, d = host(x), host(ids).astype(np.int64), host(dw)
    ds, on = np.zeros((T, E)), np.zeros((T, E))
    np.put_along_axis(ds, i, d, 1)
    np.put_along_axis(on, i, 1.0, 1)
    e = np.exp(l - l.max(1, keepdims=True))
    full = e / e.sum(1, keepdims=True) if score == "softmax" else 1 / (1 + np.exp(-l))
    share = full * on / ((full * on).sum(1, keepdims=True) + 1e-20) if renorm else full
    outer = 1 / (1 + np.exp(l)) if score == "sigmoid" else 1.0  # the sigmoid's 1 - s beside it
    # an expert's share times the sum over j of share_j (d_i - d_j)
    pairs = share[:, :, None] * share[:, None, :]
    want = outer * (pairs * (ds[:, :, None] - ds[:, None, :])).sum(2)
    size = outer * (pairs * (1 - np.eye(E)) * (np.abs(ds)[:, :, None] + np.abs(ds)[:, None, :])).sum(2)
    if renorm:  # and what the 1e-20 beside the sum leaves: of each share, and of the softmax's own sum
        total = (full * on).sum(1, keepdims=True)
        for v, sign, out in ((ds, 1, want), (np.abs(ds), -1, size)):
            left = (full * v).sum(1, keepdims=True) * 1e-20 / (total + 1e-20) ** 2
            out += outer * full * on * left / total - sign * (score == "softmax") * full * left
    close(got, want, 128 * E24 * size, dtype, "dlogits")


def test_route_bwd_more_tokens_than_a_launch_takes(torch, isc):
    """Tokens on either side of a launch's last one, and the last, as in a small call; none left out."""
    T, E, k = 2 ** 26 + 3, 4, 2
    note("route bwd many tokens", T)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((T, E), generator=g, device="cuda", dtype=torch.bfloat16)
    ids = torch.arange(k, device="cuda", dtype=torch.int32).expand(T, k).contiguous()
    dw = torch.randn((T, k), generator=g, device="cuda")
    got = isc.isc_route_bwd(dw, x, ids)
    cut = 2 ** 26 - 4
    for rows in (slice(0, 4), slice(cut - 4, cut + 4), slice(T - 4, T)):
        assert torch.equal(got[rows], isc.isc_route_bwd(dw[rows], x[rows], ids[rows])), rows
    # and every token's, by w (1 - w) (dweights_0 - dweights_1) of its two experts
    for t in range(0, T, 1 << 23):
        l, d = x[t:t + (1 << 23)].double(), dw[t:t + (1 << 23)].double()
        w = torch.sigmoid(l[:, 0] - l[:, 1])
        want = w * (1 - w) * (d[:, 0] - d[:, 1])
        size = 128 * E24 * 2 * d.abs().sum(-1) + U["bfloat16"] * want.abs()
        mine = got[t:t + (1 << 23)].double()
        assert ((mine[:, 0] - want).abs() <= size).all() and ((mine[:, 1] + want).abs() <= size).all(), t


def test_route_bwd_against_differences(torch, isc):
    """Along a direction that does not change the choice (the step is small against the gaps)."""
    note("route bwd differences")
    r = np.random.default_rng(2)
    T, E, k = 3, 10, 3
    l = np.stack([r.permutation(E) * 0.5 for _ in range(T)])
    dw, v = r.standard_normal((T, k)), r.standard_normal((T, E))
    for score in ("softmax", "sigmoid"):
        got = isc.isc_route(dev(torch, l), k, score=score)
        dl = host(isc.isc_route_bwd(dev(torch, dw), dev(torch, l), got.ids, score=score))
        step = 2.0 ** -6
        f = lambda s: (host(isc.isc_route(dev(torch, l + s * v), k, score=score).weights) * dw).sum()  # noqa: E731
        # fp32 weights err by 64 e each, the third derivative by step^2 / 6 of terms of size 1
        assert abs((f(step) - f(-step)) / (2 * step) - (dl * v).sum()) <= 64 * E24 * np.abs(dw).sum() / step + \
            step ** 2 * np.abs(dw).sum()


# ---------------------------------------------------------------- products --

def weights(torch, isc, r, E, N, K, layout, lead=None):
    """(packed, values in 64 bits) of random codes and scales."""
    codes = r.integers(0, 256, (E, N, (K + 1) // 2), dtype=np.uint8)
    scales = r.integers(119, 130, (E, N, (K + 31) // 32), dtype=np.uint8)
    values = ffn.fp4_values(codes, scales, K)
    c, s = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    if lead is None:
        c, s = c[0], s[0]
    return isc.isc_w4_pack_codes(c, s, layout, K=K), values


def mx8(torch, isc, x):
    """(tensors, values) of rows in 8 bits."""
    b = (ffn.scale_exponents(x, 448.0) + 127).astype(np.uint8)
    u = x / np.repeat(ffn.scale_values(b), 32, axis=-1)[..., : x.shape[-1]]
    q = torch.from_numpy(u).to(torch.float8_e4m3fn)
    values = ffn.mx8_values(q.view(torch.uint8).numpy(), b)
    return isc.Mx8(q.cuda(), torch.from_numpy(b).cuda().view(torch.float8_e8m0fnu)), values


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", [(1, 1), (3, 31), (16, 32), (17, 33), (5, 64), (40, 1000)])
def test_quantize(torch, isc, N, K, dtype):
    note("quantize", N, K, dtype)
    r = np.random.default_rng(N + K)
    w = dev(torch, r.standard_normal((N, K)) * 0.05, dtype)
    w[0, 0] = float("nan")
    codes, scales = isc.isc_w4_quantize(w)
    want = ffn.fp4_quantize(host(w))
    assert np.array_equal(host(scales), want[1])
    got = ffn.fp4_values(host(codes), host(scales), K)
    v = ffn.fp4_values(*want, K)
    assert ((got == v) | (np.isnan(got) & np.isnan(v))).all()
    s, t = isc.isc_w4_quantize(strided(w, 3))
    assert torch.equal(s, codes) and torch.equal(t.view(torch.uint8), scales.view(torch.uint8))


def test_quantize_in_turns(torch, isc):
    """More groups than a grid has threads."""
    E, N, K = 70, 2 ** 24, 1
    note("quantize in turns", E, N, K)
    w = torch.randint(-127, 128, (E, N, K), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda",
                      dtype=torch.int8).bfloat16()
    codes, scales = isc.isc_w4_quantize(w)
    assert w.numel() > 2 ** 30
    # each of the 255 values by itself, then all of them bit for bit
    want = [torch.from_numpy(v[:, 0]).cuda() for v in ffn.fp4_quantize(np.arange(-127.0, 128.0)[:, None])]
    for e in range(E):
        at = (w[e, :, 0].float() + 127).long()
        assert torch.equal(codes[e, :, 0], want[0][at]) and torch.equal(scales[e].view(torch.uint8)[:, 0], want[1][at]), e


PRODUCTS = [(1, 1, 1), (2, 15, 2), (1, 16, 31), (3, 17, 32), (5, 100, 33), (6, 64, 127), (8, 33, 128), (9, 130, 129),
            (16, 48, 511), (17, 20, 512), (1, 300, 513), (33, 40, 1000), (65, 70, 640), (130, 36, 300), (2, 24, 4500),
            (64, 200, 2050)]


@pytest.mark.parametrize("xtype", TYPES + ["mx8"])
@pytest.mark.parametrize("T,N,K", PRODUCTS)
def test_linear(torch, isc, T, N, K, xtype):
    note("linear", T, N, K, xtype)
    r = np.random.default_rng(T * 100 + N + K)
    w4, w = weights(torch, isc, r, 1, N, K, "tiles")
    x = r.standard_normal((T, K)) * np.exp(r.standard_normal((T, 1)))
    xd, xv = mx8(torch, isc, x) if xtype == "mx8" else (dev(torch, x, xtype), None)
    xv = host(xd) if xv is None else xv
    want, size = ffn.product(w[0], xv)
    for ytype, relu in (("float32", False), ("bfloat16", True), ("float16", False)):
        y = isc.isc_w4_linear(xd, w4, relu=relu, dtype=getattr(torch, ytype))
        assert y.shape == (T, N)
        with np.errstate(over="ignore"):
            ref = np.maximum(want, 0) if relu else want
        close(host(y), ref, (K + 64) * E24 * size, ytype, "y")
    if xtype != "mx8":
        for extra, shift in ((8, 0), (3, 1)):
            assert torch.equal(isc.isc_w4_linear(strided(xd, extra, shift), w4, dtype=torch.float32),
                               isc.isc_w4_linear(xd, w4, dtype=torch.float32))
    else:
        s = isc.Mx8(strided(xd.q.view(torch.uint8), 5, 1).view(torch.float8_e4m3fn),
                    strided(xd.scales.view(torch.uint8), 2).view(torch.float8_e8m0fnu))
        assert torch.equal(isc.isc_w4_linear(s, w4, dtype=torch.float32), isc.isc_w4_linear(xd, w4, dtype=torch.float32))


# shapes on either side of every size that the product's tiling goes by, each
# with several steps of 128 inputs for every wavefront and a last one that is not full
TILINGS = [(1, 40, 1500), (4, 40, 1500), (1, 40, 7000), (1, 8200, 1500), (6, 8200, 1500), (1, 16400, 1200), (5, 16400, 1200),
           (16, 16400, 1200), (17, 40, 1500), (20, 5000, 1500), (40, 4100, 1500), (64, 4100, 1500), (64, 8200, 1500), (60, 16400, 1200),
           (70, 16400, 1201)]


@pytest.mark.parametrize("xtype", TYPES + ["mx8"])
@pytest.mark.parametrize("T,N,K", TILINGS)
def test_linear_tilings(torch, isc, T, N, K, xtype):
    note("linear tilings", T, N, K, xtype)
    r = np.random.default_rng(T + N + K)
    w4, w = weights(torch, isc, r, 1, N, K, "tiles")
    x = r.standard_normal((T, K))
    xd, xv = mx8(torch, isc, x) if xtype == "mx8" else (dev(torch, x, xtype), None)
    xv = host(xd) if xv is None else xv
    want, size = ffn.product(w[0], xv)
    close(host(isc.isc_w4_linear(xd, w4, dtype=torch.float32)), want, (K + 64) * E24 * size, "float32", "y")


@pytest.mark.parametrize("xtype", TYPES + ["mx8"])
@pytest.mark.parametrize("T,N", [(20, 8900), (20, 13000), (40, 11000), (40, 14001), (11, 11000), (11, 14000), (90, 4100), (130, 4100),
                                 (100, 16400), (130, 7000), (130, 16400)])
def test_linear_workgroup_shapes(torch, isc, T, N, xtype):
    """Three and four tiles of outputs by two and three of columns."""
    note("linear workgroup shapes", T, N, xtype)
    r, K = np.random.default_rng(T + N), 700
    w4, w = weights(torch, isc, r, 1, N, K, "tiles")
    x = r.standard_normal((T, K))
    xd, xv = mx8(torch, isc, x) if xtype == "mx8" else (dev(torch, x, xtype), None)
    xv = host(xd) if xv is None else xv
    want, size = ffn.product(w[0], xv)
    close(host(isc.isc_w4_linear(xd, w4, dtype=torch.float32)), want, (K + 64) * E24 * size, "float32", "y")


@pytest.mark.parametrize("xtype", TYPES + ["mx8"])
@pytest.mark.parametrize("T,N,K", [(1, 5000, 4500), (5, 5000, 700), (3, 11000, 600), (5, 11000, 1500), (1, 15000, 600),
                                   (5, 17000, 1500), (1, 33000, 600), (1, 2100, 6600), (16, 8200, 4300),
                                   (16, 100, 8100), (5, 300, 9001), (16, 4200, 8200), (8, 4200, 16400)])
def test_linear_few_tokens(torch, isc, T, N, K, xtype):
    """One to four tiles of outputs a workgroup, four and eight wavefronts, rows shorter than those and longer."""
    note("linear few tokens", T, N, K, xtype)
    r = np.random.default_rng(T + N + K)
    w4, w = weights(torch, isc, r, 1, N, K, "tiles")
    x = r.standard_normal((T, K))
    xd, xv = mx8(torch, isc, x) if xtype == "mx8" else (dev(torch, x, xtype), None)
    xv = host(xd) if xv is None else xv
    want, size = ffn.product(w[0], xv)
    close(host(isc.isc_w4_linear(xd, w4, dtype=torch.float32)), want, (K + 64) * E24 * size, "float32", "y")


@pytest.mark.parametrize("xtype", ["bfloat16", "float16", "mx8"])
@pytest.mark.parametrize("T", [2, 4, 5, 60])
def test_experts_long_rows(torch, isc, T, xtype):
    """Experts' rows of several steps for every wavefront, few tokens and many."""
    note("experts long rows", T, xtype)
    r = np.random.default_rng(T)
    E, k, N, K = 5, 2, 100, 2600
    route, ids, _ = a_route(torch, isc, r, T, E, k, 0.1)
    w4, w = weights(torch, isc, r, E, N, K, "tiles", lead=E)
    x = r.standard_normal((T, K))
    xd, xv = mx8(torch, isc, x) if xtype == "mx8" else (dev(torch, x, xtype), None)
    xv = host(xd) if xv is None else xv
    want, size = ffn.routed(w, xv, ids)
    y = isc.isc_w4_linear(xd, w4, route=route, dtype=torch.float32)
    close(host(y), want, (K + 64) * E24 * size, "float32", "y")


@pytest.mark.parametrize("T,K,N", [(1, 70, 40), (3, 900, 600), (16, 5000, 520)])
def test_skip_scales(torch, isc, T, K, N):
    """Scales from 2^-127 to 2^124 and NaN ones, counts of nonzeros that end a batch early: nothing leaks from
    one group to the next, from a batch's last row to the entries behind it, or from what a 0 would meet."""
    note("skip scales", T, K, N)
    r = np.random.default_rng(K)
    codes = r.integers(0, 256, (N, (K + 1) // 2), dtype=np.uint8)
    scales = r.integers(0, 252, (N, (K + 31) // 32), dtype=np.uint8)
    x = r.standard_normal((T, K)) * (r.random((T, K)) < 0.07)
    w = ffn.fp4_values(codes, scales, K)
    pack = lambda s: isc.isc_w4_pack_codes(torch.from_numpy(codes).cuda(), torch.from_numpy(s).cuda(), "rows", K=K)  # noqa: E731
    xd = dev(torch, x)
    x = host(xd)
    # a term's own rounding is absolute below fp32's smallest normal number
    with np.errstate(over="ignore"):
        size = np.abs(x) @ np.abs(w).T
        got, want = host(isc.isc_w4_skip(xd, pack(scales), dtype=torch.float32)), x @ w.T
    fits = size < 1e38
    assert fits.any()
    assert (np.abs(got - want)[fits] <= ((K + 64) * E24 * size + K * 2.0 ** -149)[fits]).all()
    # an output's NaN group is met by a token with a nonzero there, and by no other
    scales[:, 0] = np.where(np.arange(N) % 3 == 0, 255, 127)
    scales[:, 1:] = 127
    meets = (x[:, :32] != 0).any(1)[:, None] & (np.arange(N) % 3 == 0)[None]
    assert np.array_equal(np.isnan(host(isc.isc_w4_skip(xd, pack(scales), dtype=torch.float32))), meets)


@pytest.mark.parametrize("N", [16, 48])
def test_linear_a_million_tokens(torch, isc, N):
    """The largest count of tokens, in fp32 the most columns: every one, against a product in 64 bits."""
    note("linear a million tokens", N)
    T, K = 2 ** 20, 8
    w4, w = weights(torch, isc, np.random.default_rng(N), 1, N, K, "tiles")
    x = torch.randn((T, K), generator=torch.Generator(device="cuda").manual_seed(N), device="cuda")
    v, wd = x.double(), torch.from_numpy(w[0].T.copy()).cuda()
    got = isc.isc_w4_linear(x, w4).double()
    assert ((got - v @ wd).abs() <= (K + 64) * E24 * (v.abs() @ wd.abs()) + E24 * got.abs()).all()


@pytest.mark.parametrize("xtype,T,K", [("float32", 20003, 2500), ("float16", 20003, 4090), ("bfloat16", 20003, 8190), ("mx8", 20003, 8190)])
def test_linear_laid_out_in_turns(torch, isc, xtype, T, K):
    """More of x than the workgroups that lay it out hold at a time: every token, against a product in 64 bits."""
    note("linear laid out in turns", xtype, T, K)
    r, N = np.random.default_rng(K), 40
    w4, w = weights(torch, isc, r, 1, N, K, "tiles")
    g = torch.Generator(device="cuda").manual_seed(1)
    if xtype == "mx8":
        q = torch.randint(0, 127, (T, K), generator=g, device="cuda", dtype=torch.uint8)
        q |= torch.randint(0, 2, (T, K), generator=g, device="cuda", dtype=torch.uint8) << 7
        scales = torch.randint(119, 130, (T, (K + 31) // 32), generator=g, device="cuda", dtype=torch.uint8)
        x = isc.Mx8(q.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu))
        v = x.q.double() * torch.exp2(scales.double() - 127).repeat_interleave(32, 1)[:, :K]
    else:
        x = torch.randn((T, K), generator=g, device="cuda").to(getattr(torch, xtype))
        v = x.double()
    wd = torch.from_numpy(w[0].T.copy()).cuda()
    got = isc.isc_w4_linear(x, w4, dtype=torch.float32).double()
    assert ((got - v @ wd).abs() <= (K + 64) * E24 * (v.abs() @ wd.abs()) + E24 * got.abs()).all()


# the same for the skipping product: one, two and four tests a turn, one range and many
@pytest.mark.parametrize("T,N,K", [(1, 40, 9000), (1, 8200, 33000), (3, 2000, 20000), (12, 4200, 5000), (40, 600, 3000),
                                   (700, 40, 700)])
def test_skip_cuts(torch, isc, T, N, K):
    note("skip cuts", T, N, K)
    r = np.random.default_rng(T + N + K)
    w4, w = weights(torch, isc, r, 1, N, K, "rows")
    x = np.abs(r.standard_normal((T, K))) * (r.random((T, K)) < 0.1)
    xd = dev(torch, x, "bfloat16")
    want, size = ffn.product(w[0], host(xd), skip=True)
    close(host(isc.isc_w4_skip(xd, w4, dtype=torch.float32)), want, (K + 64) * E24 * size, "float32", "y")


@pytest.mark.parametrize("xtype", TYPES)
@pytest.mark.parametrize("T,N,K", PRODUCTS)
def test_skip(torch, isc, T, N, K, xtype):
    note("skip", T, N, K, xtype)
    r = np.random.default_rng(T * 100 + N + K)
    w4, w = weights(torch, isc, r, 1, N, K, "rows")
    x = np.abs(r.standard_normal((T, K))) * (r.random((T, K)) < r.choice([0.02, 0.1, 0.5, 1.0], (T, 1)))
    x[0] = 0
    x[-1, ::3] = -0.0
    if T > 2:
        x[1, : K // 2] = 0
    xd = dev(torch, x, xtype)
    want, size = ffn.product(w[0], host(xd))
    for ytype in TYPES:
        y = isc.isc_w4_skip(xd, w4, dtype=getattr(torch, ytype))
        close(host(y), want, (K + 64) * E24 * size, ytype, "y")
    assert T == 1 or (host(y)[0] == 0).all()
    s = isc.isc_w4_skip(strided(xd, 3, 1), w4)
    assert torch.equal(s, isc.isc_w4_skip(xd, w4))


@pytest.mark.parametrize("slots", [0, 2])
def test_skip_more_tokens_than_a_launch_takes(torch, isc, slots):
    """Tokens on either side of a launch's last one, and the last, as in a small call; none left out."""
    T, N, K, E = 2 ** 20, 4224, 32, 2  # nine workgroups a token: 932067 tokens a launch
    note("skip many tokens", slots)
    r = np.random.default_rng(slots)
    w4, w = weights(torch, isc, r, E if slots else 1, N, K, "rows", lead=E if slots else None)
    g = torch.Generator(device="cuda").manual_seed(1)
    shape = (T, slots, K) if slots else (T, K)
    x = torch.relu(torch.randn(shape, generator=g, device="cuda")).bfloat16()
    route = None
    if slots:
        first = torch.randint(0, E, (T, 1), generator=g, device="cuda", dtype=torch.int32)
        route = isc.Route(torch.cat((first, 1 - first), 1), torch.rand((T, slots), generator=g, device="cuda"), None, None)
    y = isc.isc_w4_skip(x, w4, route=route)
    cut = (2 ** 32 - 1) // 512 // 9
    for rows in (slice(0, 4), slice(cut - 4, cut + 4), slice(T - 4, T)):
        part = route and isc.Route(route.ids[rows], route.weights[rows], None, None)
        small = isc.isc_w4_skip(x[rows], w4, route=part)
        # one range of inputs here, one there: the same sums
        assert torch.equal(y[rows], small), rows
    # and every token's first outputs, by a product in 64 bits
    n = 8
    wd = torch.from_numpy(w[:, :n]).cuda()
    for t in range(0, T, 1 << 18):
        v = x[t:t + (1 << 18)].double()
        v = v if slots else v[:, None]
        e = route.ids[t:t + (1 << 18)].long() if slots else torch.zeros((v.shape[0], 1), dtype=torch.long, device="cuda")
        f = route.weights[t:t + (1 << 18)].double() if slots else torch.ones((v.shape[0], 1), device="cuda").double()
        want, size = 0.0, 0.0
        for j in range(v.shape[1]):
            both = torch.stack([v[:, j] @ wd[i].t() for i in range(wd.shape[0])], 1)
            sizes = torch.stack([v[:, j].abs() @ wd[i].abs().t() for i in range(wd.shape[0])], 1)
            at = e[:, j, None, None].expand(-1, 1, n)
            want = want + f[:, j, None] * both.gather(1, at)[:, 0]
            size = size + f[:, j, None] * sizes.gather(1, at)[:, 0]
        got = y[t:t + (1 << 18), :n].double()
        assert ((got - want).abs() <= (2 * K + 64) * E24 * size + U["bfloat16"] * want.abs()).all(), t


def a_route(torch, isc, r, T, E, k, empty):
    """A route whose ids and weights are drawn: some slots empty, lists by expert."""
    ids = np.stack([r.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    ids[r.random((T, k)) < empty] = -1
    offsets, order = ffn.lists(ids, E)
    w = r.random((T, k)).astype(np.float32)
    w[ids < 0] = 0
    dv = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    return isc.Route(dv(ids), dv(w), dv(offsets), dv(order)), ids, w


@pytest.mark.parametrize("xtype", TYPES + ["mx8"])
@pytest.mark.parametrize("T,E,N", [(20, 64, 260), (100, 3, 70), (300, 8, 530), (97, 2, 530)])
def test_experts_many_rows(torch, isc, T, E, N, xtype):
    """More rows an expert than one matrix operand holds, few and many outputs."""
    note("experts many rows", T, E, N, xtype)
    r, K, k = np.random.default_rng(T + N), 300, 2
    route, ids, _ = a_route(torch, isc, r, T, E, k, 0.1)
    w4, w = weights(torch, isc, r, E, N, K, "tiles", lead=E)
    x = r.standard_normal((T, K))
    xd, xv = mx8(torch, isc, x) if xtype == "mx8" else (dev(torch, x, xtype), None)
    xv = host(xd) if xv is None else xv
    want, size = ffn.routed(w, xv, ids)
    close(host(isc.isc_w4_linear(xd, w4, route=route, dtype=torch.float32)), want, (K + 64) * E24 * size, "float32", "y")


@pytest.mark.parametrize("xtype", TYPES + ["mx8"])
@pytest.mark.parametrize("T,E,k,N,K,empty", [(1, 3, 2, 20, 70, 0.0), (5, 4, 4, 33, 128, 0.3), (40, 6, 2, 17, 600, 0.1),
                                             (100, 2, 1, 40, 64, 0.5), (3, 64, 8, 16, 520, 0.0), (4, 5, 3, 30, 96, 1.0)])
def test_experts(torch, isc, T, E, k, N, K, empty, xtype):
    note("experts", T, E, k, N, K, empty, xtype)
    r = np.random.default_rng(T + E + N)
    route, ids, wt = a_route(torch, isc, r, T, E, k, empty)
    w4, w = weights(torch, isc, r, E, N, K, "tiles", lead=E)
    x = r.standard_normal((T, K))
    xd, xv = mx8(torch, isc, x) if xtype == "mx8" else (dev(torch, x, xtype), None)
    xv = host(xd) if xv is None else xv
    want, size = ffn.routed(w, xv, ids)
    y = isc.isc_w4_linear(xd, w4, route=route, dtype=torch.float32)
    close(host(y), want, (K + 64) * E24 * size, "float32", "y")
    assert (host(y)[ids < 0] == 0).all()
    if xtype == "mx8":
        return
    # the second products, on [T, k, K] rows
    rows, rw = weights(torch, isc, r, E, N, K, "rows", lead=E)
    h = np.maximum(r.standard_normal((T, k, K)), 0) * (r.random((T, k, K)) < 0.4)
    hd = dev(torch, h, xtype)
    vals, sizes = ffn.routed(rw, host(hd), ids, skip=True)
    y = isc.isc_w4_skip(hd, rows, route=route, dtype=torch.float32)
    close(host(y), (vals * wt[..., None]).sum(1), (K * k + 64) * E24 * (sizes * wt[..., None]).sum(1), "float32", "sum")


@pytest.mark.parametrize("xtype", TYPES + ["mx8"])
@pytest.mark.parametrize("T,E,k,N,K,popular", [(100, 5, 2, 530, 2600, False), (150, 4, 2, 70, 1600, True), (24, 16, 2, 1040, 2600, False),
                                               (40, 9, 2, 1840, 1100, True), (700, 6, 3, 130, 700, False)])
def test_experts_many_long_rows(torch, isc, T, E, k, N, K, popular, xtype):
    """Several tiles of an expert's pairs, each by several steps of every wavefront; half of all pairs with one expert."""
    note("experts many long rows", T, E, k, N, K, popular, xtype)
    r = np.random.default_rng(T + N)
    ids = np.stack([r.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    if popular:
        ids[:, 0] = 1
        ids[:, 1] = np.where(r.random(T) < 0.1, -1, np.where(ids[:, 1] == 1, 0, ids[:, 1]))
    offsets, order = ffn.lists(ids, E)
    dv = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    route = isc.Route(dv(ids), torch.ones((T, k), device="cuda"), dv(offsets), dv(order))
    w4, w = weights(torch, isc, r, E, N, K, "tiles", lead=E)
    x = r.standard_normal((T, K))
    xd, xv = mx8(torch, isc, x) if xtype == "mx8" else (dev(torch, x, xtype), None)
    xv = host(xd) if xv is None else xv
    want, size = ffn.routed(w, xv, ids)
    close(host(isc.isc_w4_linear(xd, w4, route=route, dtype=torch.float32)), want, (K + 64) * E24 * size, "float32", "y")


@pytest.mark.parametrize("xtype", TYPES + ["mx8"])
@pytest.mark.parametrize("T,N,K", [(257, 700, 1500), (1000, 260, 2100), (1003, 2100, 640), (3001, 100, 900)])
def test_linear_many_tokens(torch, isc, T, N, K, xtype):
    note("linear many tokens", T, N, K, xtype)
    r = np.random.default_rng(T + N + K)
    w4, w = weights(torch, isc, r, 1, N, K, "tiles")
    x = r.standard_normal((T, K))
    xd, xv = mx8(torch, isc, x) if xtype == "mx8" else (dev(torch, x, xtype), None)
    xv = host(xd) if xv is None else xv
    want, size = ffn.product(w[0], xv)
    close(host(isc.isc_w4_linear(xd, w4, dtype=torch.float32)), want, (K + 64) * E24 * size, "float32", "y")


def test_product_values(torch, isc):
    """NaN scales and inputs that are no numbers: where the 64-bit form has them, and
    a zero of a rectified x reads no weight."""
    note("product values")
    r = np.random.default_rng(5)
    N, K = 20, 160
    codes = r.integers(0, 256, (N, K // 2), dtype=np.uint8)
    codes[7] = 0x22
    scales = r.integers(120, 130, (N, K // 32), dtype=np.uint8)
    scales[3, 2] = 255
    scales[5, 1] = 0    # 2^-127
    scales[6, 0] = 250  # 2^123
    w = ffn.fp4_values(codes, scales, K)
    c, s = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    x = np.maximum(r.standard_normal((4, K)), 0).astype(np.float32)
    x[1, 64:96] = 0   # the group of the NaN scale
    x[2, 100] = np.nan
    x[3, 130] = np.inf
    for dtype in TYPES:
        xd = dev(torch, x, dtype)
        want, size = ffn.product(w, host(xd))
        y = host(isc.isc_w4_linear(xd, isc.isc_w4_pack_codes(c, s, "tiles"), dtype=torch.float32))
        close(y, want, (K + 64) * E24 * np.nan_to_num(size, posinf=0), "float32", "linear " + dtype)
        want, size = ffn.product(w, host(xd), skip=True)
        y = host(isc.isc_w4_skip(xd, isc.isc_w4_pack_codes(c, s, "rows"), dtype=torch.float32))
        close(y, want, (K + 64) * E24 * np.nan_to_num(size, posinf=0), "float32", "skip " + dtype)
        assert np.isfinite(y[1]).all() and np.isnan(y[0, 3])


def test_no_tokens(torch, isc):
    note("no tokens")
    r = np.random.default_rng(1)
    t, _ = weights(torch, isc, r, 1, 8, 64, "tiles")
    w, _ = weights(torch, isc, r, 1, 8, 64, "rows")
    x = torch.empty((0, 64), device="cuda")
    assert isc.isc_w4_linear(x, t).shape == (0, 8) and isc.isc_w4_skip(x, w).shape == (0, 8)


def test_fp32_inputs_count_in_full(torch, isc):
    """An fp32 x enters with all its bits: 1 + 2^-23 times 1 is no other number."""
    note("fp32 in full")
    codes = torch.full((16, 1), 0x02, dtype=torch.uint8, device="cuda")  # the weights 1 and 0
    w = isc.isc_w4_pack_codes(codes, torch.full((16, 1), 127, dtype=torch.uint8, device="cuda"), "tiles")
    v = np.array([1 + 2.0 ** -23, np.finfo(np.float32).max, -(2 - 2.0 ** -23), 1 / 3], dtype=np.float32)
    x = torch.zeros((4, 2), device="cuda")
    x[:, 0] = torch.from_numpy(v).cuda()
    assert np.array_equal(isc.isc_w4_linear(x, w).cpu().numpy(), np.repeat(v[:, None], 16, 1))


@pytest.mark.parametrize("T", [1, 4, 30])
def test_small_fp32_inputs(torch, isc, T):
    """fp32 inputs from 2^-110 on enter with all their bits; below, the parts drop what is under 2^-133 (a
    bfloat16's last place), of each input less than that."""
    note("small fp32 inputs", T)
    r = np.random.default_rng(T)
    N, K = 40, 300
    codes = r.integers(0, 256, (1, N, K // 2), dtype=np.uint8)
    w = ffn.fp4_values(codes, np.full((1, N, (K + 31) // 32), 127, dtype=np.uint8), K)[0]
    w4 = isc.isc_w4_pack_codes(torch.from_numpy(codes[0]).cuda(),
                               torch.full((N, (K + 31) // 32), 127, dtype=torch.uint8, device="cuda"), "tiles")
    for low, lost in ((-110, 0.0), (-126, 2.0 ** -133), (-140, 2.0 ** -133)):
        x = (1 + r.random((T, K))) * 2.0 ** r.integers(low, low + 6, (T, K)) * r.choice([-1, 1], (T, K))
        xd = dev(torch, x)
        want, size = ffn.product(w, host(xd))
        # and what fp32 sums drop below their own last place
        bound = (K + 64) * E24 * size + lost * np.abs(w).sum(1)[None] + (K + 64) * 2.0 ** -149
        got = host(isc.isc_w4_linear(xd, w4, dtype=torch.float32))
        assert (np.abs(got - want) <= bound).all(), low


@pytest.mark.parametrize("T", [1, 4, 30])
def test_small_group_scales(torch, isc, T):
    """8-bit inputs under scale bytes from 3 on, weights under any: with all their bits; under 0, 1 and 2 an input's bits
    below 2^-133 are rounded."""
    note("small group scales", T)
    r = np.random.default_rng(T)
    N, K = 40, 320
    codes = r.integers(0, 256, (1, N, K // 2), dtype=np.uint8)
    q = (r.integers(0, 127, (T, K)) | r.integers(0, 2, (T, K)) << 7).astype(np.uint8)
    for ws, xs, lost in ((127, (3, 12), 0.0), (0, (120, 130), 0.0), (1, (140, 200), 0.0), (150, (3, 30), 0.0), (127, (0, 3), 2.0 ** -134)):
        scales = r.integers(*xs, (T, K // 32), dtype=np.uint8)
        w = ffn.fp4_values(codes, np.full((1, N, K // 32), ws, dtype=np.uint8), K)[0]
        w4 = isc.isc_w4_pack_codes(torch.from_numpy(codes[0]).cuda(),
                                   torch.full((N, K // 32), ws, dtype=torch.uint8, device="cuda"), "tiles")
        x = isc.Mx8(torch.from_numpy(q).cuda().view(torch.float8_e4m3fn), torch.from_numpy(scales).cuda().view(torch.float8_e8m0fnu))
        want, size = ffn.product(w, ffn.mx8_values(q, scales))
        bound = (K + 64) * E24 * size + lost * np.abs(w).sum(1)[None] + (K + 64) * 2.0 ** -149
        got = host(isc.isc_w4_linear(x, w4, dtype=torch.float32))
        assert (np.abs(got - want) <= bound).all(), (ws, xs)


# ------------------------------------------------- streams, graphs, offsets --

def block(isc, x, res, nw, router, up, down):
    """One block: norm, route, the experts' products."""
    n = isc.isc_rmsnorm(x, nw, residual=res, mx8=True)
    r = isc.isc_route(n.y.float() @ router, 2, score="sigmoid")
    u = isc.isc_w4_linear(n.mx8, up, route=r, relu=True)
    return n.h, r.ids, r.order, isc.isc_w4_skip(u, down, route=r)


def block_inputs(torch, isc, T, seed=0):
    r = np.random.default_rng(seed)
    D, F, E = 160, 96, 6
    up, _ = weights(torch, isc, r, E, F, D, "tiles", lead=E)
    down, _ = weights(torch, isc, r, E, D, F, "rows", lead=E)
    x, res = dev(torch, r.standard_normal((T, D)), "bfloat16"), dev(torch, r.standard_normal((T, D)), "bfloat16")
    return x, res, torch.ones(D, device="cuda", dtype=torch.bfloat16), dev(torch, r.standard_normal((D, E)) * 0.1), up, down


def test_another_stream(torch, isc):
    """Work of another stream, by the argument and as the current stream, on tensors that it waits for."""
    note("streams")
    args = block_inputs(torch, isc, 70)
    want = block(isc, *args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = block(isc, *args)
    n = isc.isc_rmsnorm(args[0], args[2], residual=args[1], stream=s)
    g = isc.isc_rmsnorm_bwd(args[0], n.h, args[2], torch.ones(70, device="cuda"), stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and torch.equal(n.h, want[0])
    assert g[0].shape == n.h.shape


@pytest.mark.parametrize("T", [3, 130])
def test_graph(torch, isc, T):
    """A captured block, replayed on new inputs with work of the program between, gives the eager results."""
    note("graph", T)
    args = block_inputs(torch, isc, T)
    x = args[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        block(isc, *args)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = block(isc, *args)
    for seed in range(4):
        x.copy_(dev(torch, np.random.default_rng(50 + seed).standard_normal(x.shape), "bfloat16"))
        want = block(isc, *args)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), seed


def test_offsets_past_32_bits(torch, isc):
    """Rows 2^30 + 64 values apart, and the last of many experts: offsets of 64 bits."""
    note("offsets")
    D, T = 96, 4
    ld = 2 ** 30 + 64
    r = np.random.default_rng(3)
    vals, w = dev(torch, r.standard_normal((T, D)), "bfloat16"), torch.ones(D, device="cuda", dtype=torch.bfloat16)
    buf = torch.zeros((T - 1) * ld + D, device="cuda", dtype=torch.bfloat16)
    far = torch.as_strided(buf, (T, D), (ld, 1))
    far.copy_(vals)
    assert torch.equal(isc.isc_rmsnorm(far, w).y, isc.isc_rmsnorm(vals, w).y)
    rs = torch.ones(T, device="cuda")
    a, b = isc.isc_rmsnorm_bwd(far, far, w, rs), isc.isc_rmsnorm_bwd(vals, vals, w, rs)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(isc.isc_route(far, 3).ids, isc.isc_route(vals, 3).ids)
    one, _ = weights(torch, isc, r, 1, 24, D, "tiles")
    assert torch.equal(isc.isc_w4_linear(far, one), isc.isc_w4_linear(vals, one))
    rows, _ = weights(torch, isc, r, 1, 24, D, "rows")
    assert torch.equal(isc.isc_w4_skip(far, rows), isc.isc_w4_skip(vals, rows))
    del buf, far
    # 600 experts of 4096 x 4096: 5 GB, only the last one's bytes are written
    N = K = 4096
    E = 600
    x = dev(torch, np.maximum(r.standard_normal((1, K)), 0), "bfloat16")
    ids, order = torch.full((1, 1), E - 1, dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32).cuda()
    offsets = torch.zeros(E + 1, dtype=torch.int32).cuda()
    offsets[E] = 1
    route = isc.Route(ids, torch.ones((1, 1), device="cuda"), offsets, order)
    for layout, call in (("tiles", isc.isc_w4_linear), ("rows", isc.isc_w4_skip)):
        one, _ = weights(torch, isc, r, 1, N, K, layout)
        n = one.data.numel()
        data = torch.empty(E * n, dtype=torch.uint8, device="cuda")
        data[-n:] = one.data
        many = isc.W4(isc.W4Desc(E, N, K, one.desc.layout), data, True)
        want = call(x, one)
        got = call(x, many, route=route) if layout == "tiles" else call(x[:, None], many, route=route)
        assert torch.equal(got.view(1, N), want), layout
        del data, many


def test_example(torch, isc):
    """The block as the example runs it, small: within bfloat16's rounding of the output and of the hidden layer."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "rectified_ffn.py")
    spec = importlib.util.spec_from_file_location("rectified_ffn", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    note("example")
    err = example.main(["--tokens", "3", "--width", "160", "--hidden", "96", "--experts", "6", "--slots", "2", "--steps", "3"])
    assert err <= 2.0 ** -8
