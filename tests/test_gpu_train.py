"""The operators that train a routed block on the GPU against their 64-bit forms.

Tolerances, from the arithmetic (u: half a unit in the last place of the
output's type relative to the value, 2^-24, 2^-11, 2^-8; e = 2^-24; size: the sum
of the magnitudes of an output's terms):
  products    n terms: (n + 64) e size for any order of fp32 additions and the
              matrix cores' aligned ones, in fp32 8 e size more for the products
              of parts that are left out, plus u |y|.  A sum over k slots: k e size.
  dw          of a sum under weights: u size more, each weighted gradient being
              rounded to its type
  dweights    a dot product of K terms, each a sum over N: (N + K + 64) e size
  orth        the 64-bit form with operands rounded to fp16 errs by some d in the
              2-norm; other roundings (fp32 sums, the state's 22 bits) make others of
              the same size: 3 d, plus u |o| for the output
"""
import ctypes
import sys

import numpy as np
import pytest

import test_oracle_train
from oracle import train

pytestmark = pytest.mark.gpu

E24 = 2.0 ** -24
U = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TYPES = ["float32", "float16", "bfloat16"]
TINY = 2.0 ** -25  # half a step of the smallest fp16 numbers
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


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


@pytest.fixture(autouse=True)
def said(request):
    print("[case]", request.node.name, flush=True)
    sys.stdout.flush()


def host(t):
    return t.cpu().double().numpy() if t.dtype.is_floating_point else t.cpu().numpy()


def dev(torch, a, dtype="float32"):
    return torch.from_numpy(np.ascontiguousarray(a)).to(getattr(torch, dtype)).cuda()


def close(got, want, size, dtype, what):
    """|got - want| <= size + u |want|."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    ok = np.abs(got - want) <= size + U[dtype] * np.abs(want) + TINY * (dtype == "float16")
    if not ok.all():
        i = tuple(np.argwhere(~ok)[0])
        raise AssertionError("%s: %d of %d off; first at %s: %r, not %r within %g" % (what, (~ok).sum(), ok.size, i, got[i], want[i],
                                                                                     np.broadcast_to(size, ok.shape)[i]))


def route(torch, isc, seed, T, k, E, empty=0.0, only=None):
    """(Route, ids): each slot another expert, some slots empty; only: the experts that are asked for."""
    r = np.random.default_rng(seed)
    among = np.arange(E) if only is None else np.asarray(only)
    ids = np.stack([r.permutation(among)[:k] for _ in range(T)]).astype(np.int32) if T else np.zeros((0, k), np.int32)
    ids[r.random(ids.shape) < empty] = -1
    weights = (r.random(ids.shape) * (ids >= 0)).astype(np.float32)
    offsets, order = train.lists(ids, E)
    return isc.Route(*(torch.from_numpy(v).cuda() for v in (ids, weights, offsets, order))), ids


def operands(torch, seed, T, k, E, K, N, dtype, shared, rectified=False):
    r = np.random.default_rng(seed + 1000)
    x = r.standard_normal((T, K) if shared else (T, k, K))
    x = np.maximum(x, 0) if rectified else x
    return dev(torch, x, dtype), dev(torch, r.standard_normal((E, N, K)) * K ** -0.5, dtype)


def check_linear(torch, isc, T, k, E, K, N, dtype, relu=False, combine=False, shared=True, empty=0.1, out=None, only=None, seed=0):
    rt, ids = route(torch, isc, seed, T, k, E, empty, only)
    x, w = operands(torch, seed, T, k, E, K, N, dtype, shared, combine)
    got = isc.isc_expert_linear(x, w, rt, relu=relu, combine=combine, dtype=None if out is None else getattr(torch, out))
    want, size = train.expert_linear(host(x), host(w), ids, relu, host(rt.weights) if combine else None)
    out = out or dtype
    assert str(got.dtype) == "torch." + out
    close(host(got), want, (K + 64 + k * combine + 8 * (dtype == "float32")) * E24 * size, out, "y")
    if not combine:
        assert (host(got)[ids < 0] == 0).all()
    again = isc.isc_expert_linear(x, w, rt, relu=relu, combine=combine, dtype=getattr(torch, out))
    assert torch.equal(got, again)


# T, k, E, K, N: one pair, few, tiles of 32, 64, 128 and 256 rows; widths within, on and past a tile's and a step's
SHAPES = [(1, 1, 1, 1, 1), (1, 2, 5, 33, 17), (3, 2, 4, 64, 64), (5, 3, 3, 70, 130), (40, 2, 3, 96, 40), (70, 2, 2, 64, 128),
          (90, 1, 2, 65, 33), (150, 2, 3, 136, 72), (33, 4, 64, 128, 96)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("form", ["relu", "combine"])
def test_linear(torch, isc, shape, dtype, form):
    check_linear(torch, isc, *shape, dtype, relu=form == "relu", combine=form == "combine", shared=form == "relu")


@pytest.mark.parametrize("dtype,out", [("bfloat16", "float32"), ("float16", "bfloat16"), ("float32", "float16")])
@pytest.mark.parametrize("shape", [(3, 2, 4, 40, 20), (200, 2, 2, 72, 48)], ids=str)
def test_linear_of_another_type_and_layout(torch, isc, shape, dtype, out):
    check_linear(torch, isc, *shape, dtype, shared=False, out=out)
    check_linear(torch, isc, *shape, dtype, combine=True, shared=True, out=out)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("K", [64, 128, 192, 264, 328])
def test_linear_by_the_largest_tiles(torch, isc, K, dtype):
    """One stage of inputs, two, three, and ends within one; experts with less than a tile's rows, more, and none."""
    T, E, N = 1500, 4, 264
    rt, ids = route(torch, isc, K, T, 2, E, 0.05, only=[0, 1, 3])
    ids = ids.copy()
    ids[40:] = np.where(ids[40:] == 3, 1 - ids[40:, ::-1].clip(0, 1), ids[40:])  # expert 3: a few rows
    offsets, order = train.lists(ids, E)
    rt = isc.Route(dev(torch, ids, "int32"), rt.weights, dev(torch, offsets, "int32"), dev(torch, order, "int32"))
    x, w = operands(torch, K, T, 2, E, K, N, dtype, True)
    # enough columns of tiles that the rule takes 256 x 256: the matrix repeated
    w = w.repeat(1, 40, 1)[:, : 40 * N]
    got = host(isc.isc_expert_linear(x, w, rt, relu=True))
    want, size = train.expert_linear(host(x), host(w[:, :N]), ids, True)
    for i in (0, 17, 39):
        close(got[..., i * N:(i + 1) * N], want, (K + 64) * E24 * size, dtype, "y, columns %d" % i)
    first = got[..., :N]
    assert all((got[..., i * N:(i + 1) * N] == first).all() for i in range(40))


def test_linear_with_experts_left_out(torch, isc):
    for dtype in TYPES:
        check_linear(torch, isc, 60, 2, 9, 72, 40, dtype, only=[2, 8])
        check_linear(torch, isc, 2, 2, 9, 72, 40, dtype, only=[2, 8], empty=0.0)
    check_linear(torch, isc, 50, 2, 3, 64, 64, "bfloat16", empty=1.0)
    check_linear(torch, isc, 50, 2, 3, 64, 64, "bfloat16", empty=1.0, combine=True)


def check_bwd(torch, isc, T, k, E, K, N, dtype, form, shared, empty=0.1, only=None, seed=0):
    rt, ids = route(torch, isc, seed, T, k, E, empty, only)
    combine = form == "combine"
    x, w = operands(torch, seed, T, k, E, K, N, dtype, shared, combine)
    y = isc.isc_expert_linear(x, w, rt, relu=True) if form == "relu" else None
    dy = dev(torch, np.random.default_rng(seed + 7).standard_normal((T, N) if combine else (T, k, N)), dtype)
    got = isc.isc_expert_linear_bwd(dy, x, w, rt, y=y, combine=combine)
    want = train.expert_linear_bwd(host(dy), host(x), host(w), ids, None if y is None else host(y),
                                   host(rt.weights) if combine else None)
    parts = 8 * (dtype == "float32")
    value, size = want["dx"]
    close(host(got.dx), value, (N + 64 + k + parts) * E24 * size, dtype, "dx")
    value, size = want["dw"]
    most = max(1, np.bincount(ids[ids >= 0], minlength=E).max()) if ids.size else 1
    close(host(got.dw), value, ((most + 64 + parts) * E24 + (U[dtype] if combine else 0)) * size
          + (TINY * most * np.abs(host(x)).max() if combine and dtype == "float16" and ids.size else 0), dtype, "dw")
    if combine:
        value, size = want["dweights"]
        close(host(got.dweights), value, (N + K + 64 + parts) * E24 * size, "float32", "dweights")
        assert (host(got.dweights)[ids < 0] == 0).all()
    else:
        assert got.dweights is None
    again = isc.isc_expert_linear_bwd(dy, x, w, rt, y=y, combine=combine)
    for a, b in zip(got, again):
        assert a is None or torch.equal(a, b)
    return got, (dy, x, w, rt, y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("form,shared", [("relu", True), ("combine", False), ("combine", True), ("plain", False)])
def test_bwd(torch, isc, shape, dtype, form, shared):
    check_bwd(torch, isc, *shape, dtype, form, shared)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("form", ["relu", "combine", "plain"])
@pytest.mark.parametrize("many,groups", [(60, 8), (80, 10), (130, 16)])  # sides of dx's tiles, of dw's: 128, 64; 256, 128; 256, 256
def test_bwd_by_larger_tiles(torch, isc, dtype, form, many, groups):
    """Wide matrices: gradients that are the same for every group of columns, since the matrices are."""
    T, k, E, K, N = 700, 2, 2, 72, 40
    rt, ids = route(torch, isc, 4, T, k, E, 0.05)
    combine = form == "combine"
    x, w = operands(torch, 4, T, k, E, K, N, dtype, not combine, combine)
    xx, ww = x.repeat(*([1] * (x.dim() - 1)), many), w.repeat(1, groups, many)
    dy = dev(torch, np.random.default_rng(9).standard_normal((T, N) if combine else (T, k, N)), dtype)
    dd = torch.cat([dy] + [torch.zeros_like(dy)] * (groups - 2) + [dy], -1)  # the first and the last group of outputs
    y = None
    if form == "relu":
        y = torch.relu(dev(torch, np.random.default_rng(2).standard_normal((T, k, N)), dtype)).repeat(1, 1, groups)
    got = isc.isc_expert_linear_bwd(dd, xx, ww, rt, y=y, combine=combine)
    want = train.expert_linear_bwd(host(dy), host(x), host(w), ids, None if y is None else host(y[..., :N]),
                                   host(rt.weights) if combine else None)
    dx, dw = host(got.dx), host(got.dw)
    value, size = want["dx"]
    for i in (0, 31, many - 1):
        close(dx[..., i * K:(i + 1) * K], 2 * value, (2 * N + 64 + k) * E24 * 2 * size, dtype, "dx, columns %d" % i)
    value, size = want["dw"]
    for j in (0, groups - 1):
        for i in (0, many - 1):
            close(dw[:, j * N:(j + 1) * N, i * K:(i + 1) * K], value,
                  ((T * k + 64) * E24 + (U[dtype] if combine else 0)) * size
                  + (TINY * T * k * np.abs(host(x)).max() if combine and dtype == "float16" else 0), dtype, "dw, group %d, %d" % (j, i))
    assert (dw[:, N:(groups - 1) * N] == 0).all()
    if combine:
        value, size = want["dweights"]
        close(host(got.dweights), 2 * many * value, (groups * N + many * K + 64) * E24 * 2 * many * size, "float32", "dweights")


@pytest.mark.parametrize("E,K", [(24, 2904), (21, 3104)])
def test_bwd_of_many_uneven_experts(torch, isc, E, K):
    """Tiles of experts in the order of their sizes: some without pairs, some of one size, E a multiple of 8 and not."""
    T, k, N = 300, 3, 304
    r = np.random.default_rng(E)
    share = np.where(np.arange(E) % 5 == 1, 0.0, 1.0 + np.arange(E) % 4 * 3)
    ids = np.stack([r.choice(E, k, replace=False, p=share / share.sum()) for _ in range(T)]).astype(np.int32)
    offsets, order = train.lists(ids, E)
    rt = isc.Route(*(torch.from_numpy(v).cuda() for v in (ids, np.ones(ids.shape, np.float32), offsets, order)))
    x, w = operands(torch, E, T, k, E, K, N, "bfloat16", True)
    dy = dev(torch, r.standard_normal((T, k, N)), "bfloat16")
    y = isc.isc_expert_linear(x, w, rt, relu=True)
    for out in (None, y):
        got = host(isc.isc_expert_linear_bwd(dy, x, w, rt, y=out, dx=False).dw)
        d = host(dy) * (1 if out is None else host(out) > 0)
        for e in range(E):
            at = ids == e
            own, rows = d[at], host(x)[np.nonzero(at)[0]]
            close(got[e], own.T @ rows, (at.sum() + 64) * E24 * (np.abs(own).T @ np.abs(rows)), "bfloat16", "dw of %d" % e)


def test_bwd_gradient_against_differences(torch, isc):
    """fp32 differences of the forward pass itself, a step of 2^-6 of it: sums are linear in each operand."""
    T, k, E, K, N = 20, 2, 3, 24, 12
    got, (dy, x, w, rt, _) = check_bwd(torch, isc, T, k, E, K, N, "float32", "combine", False)
    r = np.random.default_rng(1)
    for name, at in (("x", x), ("w", w)):
        step = dev(torch, r.standard_normal(at.shape))
        f = lambda v: (isc.isc_expert_linear(v if name == "x" else x, v if name == "w" else w, rt, combine=True).double()  # noqa: E731
                       * dy.double()).sum()
        slope = float(f(at + 2.0 ** -6 * step) - f(at - 2.0 ** -6 * step)) / 2.0 ** -5
        grad = got.dx if name == "x" else got.dw
        # 480 outputs of some K e each, over the step
        assert abs(slope - float((grad.double() * step.double()).sum())) < 2.0 ** 5 * T * N * (K + 80) * E24 * 30, name


@pytest.mark.parametrize("dtype", TYPES)
def test_bwd_asked_for_in_parts(torch, isc, dtype):
    for form in ("relu", "combine"):
        got, (dy, x, w, rt, y) = check_bwd(torch, isc, 50, 2, 3, 72, 40, dtype, form, True)
        combine = form == "combine"
        for name in ("dx", "dw") + (("dweights",) if combine else ()):
            ask = dict(dx=name == "dx", dw=name == "dw", dweights=name == "dweights")
            part = isc.isc_expert_linear_bwd(dy, x, w, rt, y=y, combine=combine, **ask)
            assert torch.equal(getattr(part, name), getattr(got, name)), name
            assert sum(v is not None for v in part) == 1


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_addresses(torch, isc, dtype):
    """Rows apart, rows off 16 bytes, views of larger tensors, broadcast gradients."""
    T, k, E, K, N = 60, 2, 3, 72, 40
    rt, ids = route(torch, isc, 3, T, k, E, 0.1)
    x, w = operands(torch, 3, T, k, E, K, N, dtype, True)
    want = isc.isc_expert_linear(x, w, rt, relu=True)
    wide = torch.full((T, K + 9), float("nan"), dtype=x.dtype, device="cuda")
    for at in (0, 1, 8, 9):
        view = wide[:, at:at + K]
        view.copy_(x)
        ww = torch.full((E, N, K + 24), float("nan"), dtype=x.dtype, device="cuda")[..., at:at + K]
        ww.copy_(w)
        assert torch.equal(isc.isc_expert_linear(view, ww, rt, relu=True), want), at
        wide.fill_(float("nan"))
    turned = w.transpose(1, 2).contiguous().transpose(1, 2)  # values of a row apart: copied first
    assert torch.equal(isc.isc_expert_linear(x, turned, rt, relu=True), want)
    one = torch.ones((), dtype=x.dtype, device="cuda")
    a = isc.isc_expert_linear_bwd(one.expand(T, k, N), x, w, rt, y=want)
    b = isc.isc_expert_linear_bwd(torch.ones_like(want), x, w, rt, y=want)
    assert torch.equal(a.dx, b.dx) and torch.equal(a.dw, b.dw)
    dy = torch.randn_like(want)
    far = torch.full((T, k, N + 7), float("nan"), dtype=x.dtype, device="cuda")[..., 3:3 + N]
    far.copy_(dy)
    a, b = (isc.isc_expert_linear_bwd(v, x, w, rt, y=want) for v in (far, dy))
    assert torch.equal(a.dx, b.dx) and torch.equal(a.dw, b.dw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [3, 90])
def test_values_that_are_not_finite_stay_in_their_rows(torch, isc, T, dtype):
    k, E, K, N = 2, 3, 72, 40
    rt, ids = route(torch, isc, 5, T, k, E, 0.2)
    x, w = operands(torch, 5, T, k, E, K, N, dtype, True)
    want = isc.isc_expert_linear(x, w, rt)
    bad = x.clone()
    bad[1, 5], bad[2, 7] = float("inf"), float("nan")
    got = isc.isc_expert_linear(bad, w, rt)
    rest = [t for t in range(T) if t not in (1, 2)]
    assert torch.equal(got[rest], want[rest])
    for t in (1, 2):
        for j in range(k):
            assert not torch.isfinite(got[t, j]).any() if ids[t, j] >= 0 else (got[t, j] == 0).all()
    gone = w.clone()
    gone[0, 3] = float("nan")  # one output of one expert
    got = isc.isc_expert_linear(x, gone, rt)
    hit = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    hit[..., 3] = rt.ids == 0
    assert torch.isnan(got[hit]).all() and torch.equal(got[~hit], want[~hit])
    # a NaN that the rectifier kept lets its gradient through, a 0 does not
    y = torch.relu(want)
    y[0, 0, 0], y[0, 0, 1] = float("nan"), 0.0
    dy = torch.ones_like(y)
    a = isc.isc_expert_linear_bwd(dy, x, w, rt, y=y)
    y[0, 0, 0] = 1.0
    b = isc.isc_expert_linear_bwd(dy, x, w, rt, y=y)
    assert torch.equal(a.dx, b.dx) and torch.equal(a.dw, b.dw)


@pytest.mark.parametrize("T", [9, 300])
def test_an_expert_twice_and_many_pairs_of_one(torch, isc, T):
    """Slots that name one expert are pairs like others; few pairs of many experts that all meet one."""
    E, K, N, k = 64, 72, 40, 3
    r = np.random.default_rng(T)
    ids = np.full((T, k), 5, np.int32)
    ids[:, 2] = r.integers(-1, E, T)
    offsets, order = train.lists(ids, E)
    weights = (r.random(ids.shape) * (ids >= 0)).astype(np.float32)
    rt = isc.Route(*(torch.from_numpy(v).cuda() for v in (ids, weights, offsets, order)))
    x, w = operands(torch, T, T, k, E, K, N, "bfloat16", True)
    for combine in (False, True):
        want, size = train.expert_linear(host(x), host(w), ids, False, weights.astype(np.float64) if combine else None)
        close(host(isc.isc_expert_linear(x, w, rt, combine=combine)), want, (K + 64 + k) * E24 * size, "bfloat16", "y")
    dy = dev(torch, r.standard_normal((T, k, N)), "bfloat16")
    g = isc.isc_expert_linear_bwd(dy, x, w, rt)
    there = (ids >= 0)[..., None]
    d, xs = host(dy) * there, host(x)
    back = np.einsum("tjn,tjnk->tjk", d, host(w)[ids.clip(0)])
    size = np.einsum("tjn,tjnk->tjk", np.abs(d), np.abs(host(w))[ids.clip(0)])
    close(host(g.dx), back.sum(1), (N + 64 + k) * E24 * size.sum(1), "bfloat16", "dx")
    dw, dws = np.zeros((E, N, K)), np.zeros((E, N, K))
    for j in range(k):
        np.add.at(dw, ids[:, j].clip(0), d[:, j, :, None] * xs[:, None, :])
        np.add.at(dws, ids[:, j].clip(0), np.abs(d[:, j, :, None] * xs[:, None, :]))
    close(host(g.dw), dw, (T * k + 64) * E24 * dws, "bfloat16", "dw")


@pytest.mark.parametrize("T", [5, 400])
def test_weights_beyond_32_bits(torch, isc, T):
    """2^32 weights and more: the last expert's products and gradients as those of a call on it alone."""
    E, N, K = 9, 21848, 21848
    ids = np.full((T, 1), E - 1, np.int32)
    rt = isc.Route(*(dev(torch, v, "int32") if v.dtype != np.float32 else dev(torch, v)
                     for v in (ids, np.ones((T, 1), np.float32), *train.lists(ids, E))))
    only = isc.Route(*(dev(torch, v, "int32") if v.dtype != np.float32 else dev(torch, v)
                       for v in (ids * 0, np.ones((T, 1), np.float32), *train.lists(ids * 0, 1))))
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, K), generator=g, device="cuda").bfloat16()
    w = torch.zeros((E, N, K), dtype=torch.bfloat16, device="cuda")
    assert w.numel() > 2 ** 32
    w[-1] = torch.randn((N, K), generator=g, device="cuda") * K ** -0.5
    y = isc.isc_expert_linear(x, w, rt)
    alone = w[-1:].clone()
    rows = torch.arange(0, N, 311, device="cuda")
    want = (x.double() @ alone[0, rows].double().t())[:, None]
    size = (x.double().abs() @ alone[0, rows].double().abs().t())[:, None]
    close(host(y[..., rows]), host(want), (K + 64) * E24 * host(size), "bfloat16", "y")
    got, ref = isc.isc_expert_linear_bwd(y, x, w, rt), isc.isc_expert_linear_bwd(y, x, alone, only)
    cols = torch.arange(0, K, 311, device="cuda")
    back = y[:, 0].double() @ alone[0, :, cols].double()
    size = y[:, 0].double().abs() @ alone[0, :, cols].double().abs()
    close(host(got.dx[:, cols]), host(back), (N + 64) * E24 * host(size), "bfloat16", "dx")
    assert torch.equal(got.dw[-1], ref.dw[0]) and all((part == 0).all() for part in got.dw[:-1])


def test_fp32_over_its_range(torch, isc):
    """Magnitudes from 2^-60 to 2^60, and the largest there are."""
    T, k, E, K, N = 70, 1, 2, 64, 32
    rt, ids = route(torch, isc, 6, T, k, E, 0.0)
    r = np.random.default_rng(6)
    for lo, hi in ((-60, 0), (-20, 20), (0, 60)):
        x = dev(torch, r.standard_normal((T, K)) * 2.0 ** r.integers(lo, hi, (T, K)))
        w = dev(torch, r.standard_normal((E, N, K)))
        want, size = train.expert_linear(host(x), host(w), ids)
        close(host(isc.isc_expert_linear(x, w, rt)), want, (K + 72) * E24 * size, "float32", "2^%d to 2^%d" % (lo, hi))
    x = torch.zeros((T, K), device="cuda")
    x[:, 3] = torch.finfo(torch.float32).max
    w = torch.full((E, N, K), 1.0, device="cuda")
    assert (isc.isc_expert_linear(x, w, rt) == torch.finfo(torch.float32).max).all()


def test_no_tokens(torch, isc):
    for dtype in TYPES:
        rt, _ = route(torch, isc, 0, 0, 2, 3)
        x, w = operands(torch, 0, 0, 2, 3, 40, 24, dtype, True)
        assert isc.isc_expert_linear(x, w, rt).shape == (0, 2, 24)
        assert isc.isc_expert_linear(x, w, rt, combine=True).shape == (0, 24)
        g = isc.isc_expert_linear_bwd(x.new_empty(0, 24), x, w, rt, combine=True)
        assert g.dx.shape == (0, 40) and g.dweights.shape == (0, 2) and (g.dw == 0).all() and g.dw.shape == w.shape


def test_lists_out_of_range_touch_nothing_else(torch, isc):
    """Offsets and pairs that no route has are passed over: what the good ones say is computed."""
    T, k, E, K, N = 40, 2, 3, 64, 64
    for tokens in (T, 3):
        rt, ids = route(torch, isc, 8, tokens, k, E, 0.0)
        x, w = operands(torch, 8, tokens, k, E, K, N, "bfloat16", True)
        want = isc.isc_expert_linear(x, w, rt)
        order = rt.order.clone()
        lost = int(order[1])
        order[1] = 10 ** 9
        offsets = rt.offsets.clone()
        offsets[0], offsets[E] = -5, 10 ** 9
        got = isc.isc_expert_linear(x, w, isc.Route(rt.ids, rt.weights, offsets, order))
        keep = torch.ones(tokens * k, dtype=torch.bool, device="cuda")
        keep[lost] = False
        assert torch.equal(got.view(-1, N)[keep], want.view(-1, N)[keep])


@pytest.mark.parametrize("form", ["relu", "combine", "plain"])
def test_a_place_without_a_pair_adds_nothing(torch, isc, form):
    """Weight gradients of lists with a hole, in a workspace of NaN."""
    T, k, E, K, N = 60, 2, 3, 64, 72
    combine = form == "combine"
    rt, ids = route(torch, isc, 11, T, k, E, 0.1)
    x, w = operands(torch, 11, T, k, E, K, N, "bfloat16", not combine)
    dy = dev(torch, np.random.default_rng(12).standard_normal((T, N) if combine else (T, k, N)), "bfloat16")
    y = isc.isc_expert_linear(x, w, rt, relu=True) if form == "relu" else None
    order = rt.order.clone()
    lost = int(order[1])
    order[1] = 10 ** 9
    n = ctypes.c_size_t()
    d = isc.ExpertDesc(E, N, K, 2, k, not combine)
    assert isc.lib().isc_expert_linear_bwd_workspace_size(d, T, form == "relu", combine, n) == 0
    ws = torch.full((n.value,), 255, dtype=torch.uint8, device="cuda")
    got = isc.isc_expert_linear_bwd(dy, x, w, isc.Route(rt.ids, rt.weights, rt.offsets, order), y=y, combine=combine,
                                    dx=False, dweights=False, ws=ws)
    ids = ids.copy()
    ids.reshape(-1)[lost] = -1
    want = train.expert_linear_bwd(host(dy), host(x), host(w), ids, None if y is None else host(y),
                                   host(rt.weights) if combine else None)
    value, size = want["dw"]
    close(host(got.dw), value, ((T * k + 64) * E24 + (U["bfloat16"] if combine else 0)) * size, "bfloat16", "dw")


# ------------------------------------------------------------ orthogonalize --

def gradient(seed, B, M, N, rank):
    r = np.random.default_rng(seed)
    g = r.standard_normal((B, M, N)) * (0.1 if rank else 1.0)
    return (g + (r.standard_normal((B, M, rank)) @ r.standard_normal((B, rank, N)) if rank else 0.0)) * 1e-3


def check_orth(torch, isc, g, out, coefficients=None, steps=5, eps=1e-7, **kw):
    coefficients = [COEFFICIENTS] * steps if coefficients is None else coefficients
    got = isc.isc_orthogonalize(g, steps=steps, coefficients=tuple(coefficients), eps=eps, dtype=getattr(torch, out), **kw)
    assert got.shape == g.shape and str(got.dtype) == "torch." + out
    flat, each = host(got).reshape(-1, *g.shape[-2:]), host(g).reshape(-1, *g.shape[-2:])
    for i, (o, m) in enumerate(zip(flat, each)):
        exact, rounded = (train.orthogonalize(m, coefficients, eps, v) for v in (False, True))
        allowed = 3 * np.linalg.norm(rounded - exact) + U[out] * np.linalg.norm(exact) + TINY * o.size ** 0.5
        assert np.linalg.norm(o - exact) <= allowed, (i, np.linalg.norm(o - exact), allowed)
    assert torch.equal(got, isc.isc_orthogonalize(g, steps=steps, coefficients=tuple(coefficients), eps=eps,
                                                  dtype=getattr(torch, out)))
    return got


# one row, one column, less than an operand, off and on tiles' edges, long and narrow (A in parts), several
MATRICES = [(1, 1, 1), (1, 1, 9), (2, 9, 1), (1, 7, 40), (2, 64, 64), (1, 65, 130), (3, 130, 65), (1, 33, 1030), (2, 1030, 33),
            (1, 8, 4096), (1, 200, 328), (2, 260, 100)]


@pytest.mark.parametrize("dtype,out", [("bfloat16", "bfloat16"), ("float32", "float16"), ("float16", "bfloat16")])
@pytest.mark.parametrize("shape", MATRICES, ids=str)
def test_orthogonalize(torch, isc, shape, dtype, out):
    check_orth(torch, isc, dev(torch, gradient(1, *shape, 0), dtype), out)
    if min(shape[1:]) > 8:
        check_orth(torch, isc, dev(torch, gradient(2, *shape, 3), dtype), out)


@pytest.mark.parametrize("shape,many", [((1, 300, 200), 110), ((1, 200, 300), 100), ((1, 300, 520), 90), ((1, 520, 300), 90)], ids=str)
def test_orthogonalize_by_larger_tiles(torch, isc, shape, many):
    """Tiles of 128 and 256 sides, which take many matrices: the same one many times, one other at the end."""
    g = dev(torch, np.concatenate([gradient(3, *shape, 5), gradient(4, *shape, 0)]), "bfloat16")
    stack = torch.cat([g[:1].expand(many, -1, -1), g[1:]])
    got = isc.isc_orthogonalize(stack)
    check_orth(torch, isc, stack[-2:], "bfloat16")
    for i in (0, -1):
        exact, rounded = (train.orthogonalize(host(stack[i]), [COEFFICIENTS] * 5, 1e-7, v) for v in (False, True))
        allowed = 3 * np.linalg.norm(rounded - exact) + U["bfloat16"] * np.linalg.norm(exact)
        assert np.linalg.norm(host(got[i]) - exact) <= allowed
    assert all(torch.equal(got[i], got[0]) for i in range(many))


def test_orthogonalize_steps_and_coefficients(torch, isc):
    g = dev(torch, gradient(5, 1, 90, 150, 4)[0], "bfloat16")
    own = [(4.0, -6.5, 3.0), (3.5, -5.0, 2.1), (1.875, -1.25, 0.375)]
    check_orth(torch, isc, g, "bfloat16", own, steps=3)
    for steps in (1, 2, 8):
        check_orth(torch, isc, g, "float16", steps=steps)
    check_orth(torch, isc, g, "bfloat16", [(1.5, -0.5, 0.0)] * 4, steps=4)  # the cubic iteration
    check_orth(torch, isc, g, "bfloat16", [(1.0, 0.0, 0.0)], steps=1)       # none
    one = isc.isc_orthogonalize(g, steps=3, coefficients=COEFFICIENTS)
    assert torch.equal(one, isc.isc_orthogonalize(g, steps=3, coefficients=[list(COEFFICIENTS)] * 3))


def test_orthogonalize_strides_scale_and_shapes(torch, isc):
    m = gradient(6, 4, 40, 56, 3)
    for dtype in TYPES:
        g = dev(torch, m, dtype)
        want = isc.isc_orthogonalize(g)
        assert torch.equal(isc.isc_orthogonalize(g.view(2, 2, 40, 56)).view(4, 40, 56), want)
        assert torch.equal(isc.isc_orthogonalize(g[2]), want[2])
        wide = torch.full((4, 40, 61), float("nan"), dtype=g.dtype, device="cuda")[..., 3:59]
        wide.copy_(g)
        assert torch.equal(isc.isc_orthogonalize(wide), want)
        assert torch.equal(isc.isc_orthogonalize(g.transpose(1, 2).contiguous().transpose(1, 2)), want)
    # fp32 gradients of any scale: squares leave fp32's range
    for scale in (1e-25, 1e25):
        check_orth(torch, isc, dev(torch, m[0] * scale), "bfloat16", eps=0.0)
    check_orth(torch, isc, dev(torch, m[0] * 1e-9), "bfloat16")  # a norm beside eps


@pytest.mark.parametrize("shape", [(64, 70), (70, 64), (65, 72), (72, 65), (300, 200)], ids=str)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_orthogonalize_at_the_ends_of_the_range(torch, isc, shape, dtype):
    """A power of two scales a norm and its inverse exactly, also where the inverse is beyond fp32."""
    g = dev(torch, np.random.default_rng(8).integers(-7, 8, shape), dtype)
    want = isc.isc_orthogonalize(g, eps=0.0)
    assert torch.isfinite(want).all()
    for power in (-133, -110, 100, 124):
        scaled = torch.ldexp(g.double(), torch.tensor(power, device="cuda")).to(g.dtype)
        assert (scaled != 0).sum() == (g != 0).sum()
        assert torch.equal(isc.isc_orthogonalize(scaled, eps=0.0), want), power


@pytest.mark.parametrize("shape", [(64, 520), (72, 464)], ids=str)
def test_orthogonalize_beyond_32_bits(torch, isc, shape):
    """2^31 values and more in a stack: the last matrix as the first."""
    M, N = shape
    many = 2 ** 31 // (M * N) + 8
    g = dev(torch, gradient(9, 1, M, N, 4)[0], "bfloat16")
    got = isc.isc_orthogonalize(g.expand(many, M, N).contiguous(), steps=2)
    assert got.numel() > 2 ** 31
    assert all((part == got[0]).all() for part in got.split(4096))
    check_orth(torch, isc, g, "bfloat16", steps=2)
    exact, rounded = (train.orthogonalize(host(g), [COEFFICIENTS] * 2, 1e-7, v) for v in (False, True))
    allowed = 3 * np.linalg.norm(rounded - exact) + U["bfloat16"] * np.linalg.norm(exact)
    assert np.linalg.norm(host(got[-1]) - exact) <= allowed


def test_orthogonalize_zeros_and_values_that_are_not_finite(torch, isc):
    g = dev(torch, gradient(7, 5, 40, 24, 0), "bfloat16")
    want = isc.isc_orthogonalize(g)
    g[1] = 0
    g[2, 3, 4] = float("inf")
    g[3, 39, 23] = float("nan")
    got = isc.isc_orthogonalize(g)
    assert (got[1] == 0).all() and torch.isnan(got[2]).all() and torch.isnan(got[3]).all()
    assert torch.equal(got[0], want[0]) and torch.equal(got[4], want[4])
    assert isc.isc_orthogonalize(g[:0]).shape == (0, 40, 24)


# ------------------------------------------------------- together, streams --

def step(torch, isc, x, router, up, down, dout):
    """A routed block's training step: forward, gradients, orthogonalised updates."""
    r = isc.isc_route(x.float() @ router, 2, score="sigmoid")
    u = isc.isc_expert_linear(x, up, r, relu=True)
    out = isc.isc_expert_linear(u, down, r, combine=True)
    g2 = isc.isc_expert_linear_bwd(dout, u, down, r, combine=True)
    g1 = isc.isc_expert_linear_bwd(g2.dx, x, up, r, y=u)
    dl = isc.isc_route_bwd(g2.dweights, x.float() @ router, r.ids, score="sigmoid")
    return out, g1.dx, g1.dw, g2.dw, dl, isc.isc_orthogonalize(g1.dw), isc.isc_orthogonalize(g2.dw)


def block(torch, seed, T=40, D=64, F=96, E=4):
    g = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return (draw(T, D).bfloat16(), draw(D, E) * D ** -0.5, (draw(E, F, D) * D ** -0.5).bfloat16(),
            (draw(E, D, F) * F ** -0.5).bfloat16(), draw(T, D).bfloat16())


def test_a_training_step(torch, isc):
    """Against autograd on the same values in 64 bits: bfloat16 roundings of u, of its gradient and of the results."""
    x, router, up, down, dout = block(torch, 1)
    out, dx, dup, ddown, dl, ou, od = step(torch, isc, x, router, up, down, dout)
    r = isc.isc_route(x.float() @ router, 2, score="sigmoid")
    xd, upd, dnd = (v.double().requires_grad_(True) for v in (x, up, down))
    logits = (x.float() @ router).double().requires_grad_(True)
    ids = r.ids.long()
    s = torch.sigmoid(torch.gather(logits, 1, ids))
    wts = s / s.sum(-1, keepdim=True)
    u = torch.relu((upd[ids] * xd[:, None, None, :]).sum(-1))
    y = ((dnd[ids] * u[:, :, None, :]).sum(-1) * wts[..., None]).sum(1)
    (y * dout.double()).sum().backward()
    y = y.detach()
    for name, got, want in (("out", out, y), ("dx", dx, xd.grad), ("dup", dup, upd.grad), ("ddown", ddown, dnd.grad),
                            ("dlogits", dl, logits.grad)):
        off = float((got.double() - want).norm() / want.norm())
        # three roundings in turn of 2^-9 at most, in the 2-norm; the rectifier's border moves by one of them
        assert off < 4 * 2.0 ** -8, (name, off)
    assert torch.equal(ou, isc.isc_orthogonalize(dup)) and torch.equal(od, isc.isc_orthogonalize(ddown))


def test_streams(torch, isc):
    x, router, up, down, dout = block(torch, 2)
    want = step(torch, isc, x, router, up, down, dout)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            outs.append(step(torch, isc, x, router, up, down, dout))
    r = isc.isc_route(x.float() @ router, 2, score="sigmoid")
    torch.cuda.synchronize()
    named = isc.isc_expert_linear(x, up, r, relu=True, stream=streams[0])
    other = isc.isc_orthogonalize(want[2], stream=streams[1])
    torch.cuda.synchronize()
    for got in outs:
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    assert torch.equal(other, want[5]) and named.shape == (40, 2, 96)


def test_graphs(torch, isc):
    """Captured once, replayed on other inputs, with eager work in between; two graphs, and kernels first met in one."""
    a = block(torch, 3)
    inputs = [v.clone() for v in a]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(torch, isc, *inputs)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(torch, isc, *inputs)
        graphs.append((graph, out))
    tall = torch.randn((70, 20), device="cuda").half()
    alone = torch.cuda.CUDAGraph()
    with torch.cuda.graph(alone):
        first = isc.isc_orthogonalize(tall, steps=2)
    for seed in (3, 4, 5, 6):
        for to, frm in zip(inputs, block(torch, seed)):
            to.copy_(frm)
        want = step(torch, isc, *[v.clone() for v in inputs])
        for graph, out in graphs:
            graph.replay()
            torch.cuda.synchronize()
            for got, w in zip(out, want):
                assert torch.equal(got, w), seed
        alone.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, isc.isc_orthogonalize(tall, steps=2))


def test_workspace_given(torch, isc):
    """A caller's workspace, with anything in it, and behind its end nothing is written."""
    x, router, up, down, dout = block(torch, 4)
    r = isc.isc_route(x.float() @ router, 2, score="sigmoid")
    E, F, D = up.shape
    n = ctypes.c_size_t()
    d = isc.ExpertDesc(E, F, D, 2, 2, 1)

    def room(size):
        ws = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
        return ws, ws[:size]

    assert isc.lib().isc_expert_linear_workspace_size(d, 40, 0, n) == 0
    whole, ws = room(n.value)
    want = isc.isc_expert_linear(x, up, r, relu=True)
    assert torch.equal(isc.isc_expert_linear(x, up, r, relu=True, ws=ws), want) and (whole[n.value:] == 255).all()
    assert isc.lib().isc_expert_linear_bwd_workspace_size(d, 40, 1, 0, n) == 0
    whole, ws = room(n.value)
    dy = torch.randn_like(want)
    got, ref = (isc.isc_expert_linear_bwd(dy, x, up, r, y=want, ws=w) for w in (ws, None))
    assert torch.equal(got.dx, ref.dx) and torch.equal(got.dw, ref.dw) and (whole[n.value:] == 255).all()
    d = isc.ExpertDesc(E, D, F, 2, 2, 0)
    for name, query, args in (("linear", "isc_expert_linear_workspace_size", (40, 1)),
                              ("bwd", "isc_expert_linear_bwd_workspace_size", (40, 0, 1))):
        assert getattr(isc.lib(), query)(d, *args, n) == 0
        whole, ws = room(n.value)
        if name == "linear":
            assert torch.equal(isc.isc_expert_linear(want, down, r, combine=True, ws=ws), isc.isc_expert_linear(want, down, r, combine=True))
        else:
            got, ref = (isc.isc_expert_linear_bwd(dout, want, down, r, combine=True, ws=w) for w in (ws, None))
            assert all(torch.equal(p, q) for p, q in zip(got, ref))
        assert (whole[n.value:] == 255).all()
    for shape in ((3, 40, 24), (1, 8, 4096)):
        assert isc.lib().isc_orthogonalize_workspace_size(*shape, n) == 0
        whole, ws = room(n.value)
        g = torch.randn(shape, device="cuda")
        assert torch.equal(isc.isc_orthogonalize(g, ws=ws), isc.isc_orthogonalize(g)) and (whole[n.value:] == 255).all()


def test_binding_refusals(torch, isc):
    x, router, up, down, dout = block(torch, 5)
    r = isc.isc_route(x.float() @ router, 2)
    bare = isc.isc_route(x.float() @ router, 2, lists=False)
    u = isc.isc_expert_linear(x, up, r, relu=True)
    for call in (lambda: isc.isc_expert_linear(x, up, bare), lambda: isc.isc_expert_linear(x, up[0], r),
                 lambda: isc.isc_expert_linear(x[:5], up, r), lambda: isc.isc_expert_linear(x.float(), up, r),
                 lambda: isc.isc_expert_linear(x, up[:3], r), lambda: isc.isc_expert_linear(x[:, :5], up, r),
                 lambda: isc.isc_expert_linear(x.cpu(), up, r), lambda: isc.isc_expert_linear_bwd(dout, x, up, r),
                 lambda: isc.isc_expert_linear_bwd(u, x, up, r, y=u[:1]), lambda: isc.isc_expert_linear_bwd(u, x, up, r, dweights=True),
                 lambda: isc.isc_expert_linear_bwd(u, x, up, r, dx=False, dw=False),
                 lambda: isc.isc_expert_linear_bwd(dout, u, down, r, y=u, combine=True), lambda: isc.isc_orthogonalize(x[0]),
                 lambda: isc.isc_orthogonalize(x, coefficients=(1, 2)), lambda: isc.isc_orthogonalize(x, steps=2, coefficients=[(1, 0, 0)])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: isc.isc_expert_linear(x.int(), up, r), lambda: isc.isc_expert_linear(x, up, r, dtype=torch.float64),
                 lambda: isc.isc_orthogonalize(x, dtype=torch.float32), lambda: isc.isc_orthogonalize(x.double())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: isc.isc_expert_linear(x, up, r, relu=True, combine=True), lambda: isc.isc_orthogonalize(x, steps=0),
                 lambda: isc.isc_orthogonalize(x, coefficients=(30.0, 0.0, 0.0)), lambda: isc.isc_orthogonalize(x, eps=-1.0),
                 lambda: isc.isc_expert_linear(x, up, r, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(isc.IscError):
            call()


def test_the_example_runs_and_its_gradients_hold(torch, isc):
    import os
    import runpy
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    main = runpy.run_path(os.path.join(root, "examples", "trained_experts.py"))["main"]
    # roundings to bfloat16 of the hidden layer, its gradient and the results: four of 2^-8 at most, in the 2-norm
    assert main(["--tokens", "64", "--width", "64", "--hidden", "96", "--experts", "8", "--steps", "3"]) < 4 * 2.0 ** -8


@pytest.mark.parametrize("M,N", [(128, 1024), (1024, 128), (777, 1155)])
def test_an_empty_stack_of_long_matrices(torch, isc, M, N):
    """Shapes whose sums come in parts."""
    for dtype in TYPES:
        got = isc.isc_orthogonalize(torch.empty((0, M, N), dtype=getattr(torch, dtype), device="cuda"))
        assert got.shape == (0, M, N)


def listed(ids, offsets, order, E):
    """ids with -1 for every pair that no place of its own expert's holds."""
    flat, at = ids.reshape(-1), np.full(ids.size, -1, dtype=ids.dtype)
    for i, p in enumerate(order):
        if 0 <= p < flat.size and 0 <= flat[p] < E and offsets[flat[p]] <= i < offsets[flat[p] + 1]:
            at[p] = flat[p]
    return at.reshape(ids.shape)


def disturbed(torch, isc, what, seed, T, k, E):
    """A route whose lists and ids do not agree, and the experts that are left."""
    rt, ids = route(torch, isc, seed, T, k, E, 0.1)
    ids, order, offsets = ids.copy(), host(rt.order).copy(), host(rt.offsets)
    weights = host(rt.weights).astype(np.float32)
    if what == "hole":            # pairs that no place holds
        order[[0, int(offsets[-1]) - 1]] = (10 ** 9, -1)
    elif what == "taken away":    # pairs whose expert was taken away after the lists were made
        for p in order[[0, int(offsets[-1]) - 1]]:
            ids.reshape(-1)[p] = (-1, E)[p % 2]
            weights.reshape(-1)[p] = np.nan
    else:                         # pairs among another expert's
        order[[0, int(offsets[-1]) - 1]] = order[[int(offsets[-1]) - 1, 0]]
    left = listed(ids, offsets, order, E)
    assert 0 < (left >= 0).sum() < (host(rt.ids) >= 0).sum()
    return isc.Route(*(torch.from_numpy(np.ascontiguousarray(v)).cuda() for v in (ids, weights, offsets, order))), left


def nothing_in_it(torch, isc, query, *args):
    """A workspace of NaN."""
    n = ctypes.c_size_t()
    assert getattr(isc.lib(), query)(*args, n) == 0
    return torch.full((n.value,), 255, dtype=torch.uint8, device="cuda")


def leave_nan(torch, *like):
    """Memory that the next tensors of these sizes take has NaN in it."""
    for t in [torch.full_like(t, float("nan")) for t in like]:
        del t


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("what", ["hole", "taken away", "another's"])
@pytest.mark.parametrize("T,E", [(6, 5), (25, 20), (160, 81), (40, 3), (400, 3)])  # few pairs; tiles of 32 and of 64 rows
def test_lists_that_ids_do_not_agree_with(torch, isc, T, E, what, dtype):
    """A pair is computed where its own expert's list has it; the others are empty slots, and nothing that a
    workspace or an output held before is in a result."""
    k, K, N = 2, 72, 104
    code = 0 if dtype == "float32" else 2
    parts = 8 * (dtype == "float32")
    rt, left = disturbed(torch, isc, what, 21, T, k, E)
    weights = np.where(left >= 0, host(rt.weights), 0.0)
    for shared in (True, False):
        x, w = operands(torch, 21, T, k, E, K, N, dtype, shared)
        desc = isc.ExpertDesc(E, N, K, code, k, shared)
        for form in ("plain", "relu", "combine"):
            combine, relu = form == "combine", form == "relu"
            want, size = train.expert_linear(host(x), host(w), left, relu, weights if combine else None)
            ws = nothing_in_it(torch, isc, "isc_expert_linear_workspace_size", desc, T, combine)
            leave_nan(torch, x.new_empty(want.shape))
            got = isc.isc_expert_linear(x, w, rt, relu=relu, combine=combine, ws=ws)
            close(host(got), want, (K + 64 + k * combine + parts) * E24 * size, dtype, "y")
            if not combine:
                assert (host(got)[left < 0] == 0).all()
            dy = dev(torch, np.random.default_rng(5).standard_normal(want.shape), dtype)
            ws = nothing_in_it(torch, isc, "isc_expert_linear_bwd_workspace_size", desc, T, relu, combine)
            leave_nan(torch, x, w, rt.weights)
            grads = isc.isc_expert_linear_bwd(dy, x, w, rt, y=got if relu else None, combine=combine, ws=ws)
            want = train.expert_linear_bwd(host(dy), host(x), host(w), left, host(got) if relu else None, weights if combine else None)
            value, size = want["dx"]
            close(host(grads.dx), value, (N + 64 + k + parts) * E24 * size, dtype, "dx")
            value, size = want["dw"]
            close(host(grads.dw), value, ((T * k + 64 + parts) * E24 + (U[dtype] if combine else 0)) * size, dtype, "dw")
            if combine:
                value, size = want["dweights"]
                close(host(grads.dweights), value, (N + K + 64 + parts) * E24 * size, "float32", "dweights")
                assert (host(grads.dweights)[left < 0] == 0).all()
                alone = isc.isc_expert_linear_bwd(dy, x, w, rt, combine=True, dx=False, dw=False,
                                                  ws=nothing_in_it(torch, isc, "isc_expert_linear_bwd_workspace_size", desc, T, 0, 1))
                assert torch.equal(alone.dweights, grads.dweights)


def errs_as_stated(torch, isc, shape, steps, frobenius, spectral, many):
    """Against the exact result, by the header's figures beside the rounding to fp16."""
    g = np.stack(list(test_oracle_train.draws(*shape, many)))
    got = host(isc.isc_orthogonalize(dev(torch, g), steps=steps, dtype=torch.float16))
    for o, m in zip(got, g.astype(np.float32)):
        exact = train.orthogonalize(m, [COEFFICIENTS] * steps, 1e-7)
        own = U["float16"] * np.linalg.norm(exact) + TINY * o.size ** 0.5
        off = np.linalg.norm(o - exact)
        assert off <= frobenius * np.linalg.norm(exact) + own, off / np.linalg.norm(exact)
        assert np.linalg.norm(o - exact, 2) <= spectral * np.linalg.norm(exact, 2) + own


@pytest.mark.parametrize("steps,frobenius,spectral", test_oracle_train.ERRORS)
@pytest.mark.parametrize("shape", [(65, 65), (65, 300), (100, 100), (130, 66), (200, 300), (520, 600)], ids=str)
def test_orthogonalize_errs_as_stated(torch, isc, shape, steps, frobenius, spectral):
    errs_as_stated(torch, isc, shape, steps, frobenius, spectral, 14 if max(shape) < 200 else 3)


@pytest.mark.parametrize("steps,frobenius,spectral", test_oracle_train.SMALL_ERRORS)
@pytest.mark.parametrize("shape", [(1, 1), (2, 2), (2, 3), (3, 5), (5, 3), (1, 40), (8, 8), (16, 300), (500, 32), (64, 64), (64, 300), (130, 64),
                                   (2100, 64)], ids=str)
def test_orthogonalize_small_sides_err_as_stated(torch, isc, shape, steps, frobenius, spectral):
    errs_as_stated(torch, isc, shape, steps, frobenius, spectral, 28 if max(shape) < 200 else 5)


# Calls by tiles of 128 and 256 that need matrices so wide: 1400 pairs of two experts, K and N given as
# (inputs, how often they are repeated); the tile's kernel is the one whose name has `kernel`.
WIDE = {"float32": [("F32ELb0E.*Li128ELi128E", (72, 1), (40, 30))],
        "bfloat16": [("BF16ELb0E.*Li128ELi128E", (71, 1), (33, 90)), ("BF16ELb1E.*Li128ELi128E", (72, 1), (40, 71)),
                     ("BF16ELb1E.*Li256ELi256E", (72, 1), (40, 140))],
        "float16": [("F16ELb0E.*Li128ELi128E", (71, 1), (33, 90)), ("F16ELb1E.*Li128ELi128E", (72, 1), (40, 71)),
                    ("F16ELb1E.*Li256ELi256E", (72, 1), (40, 140))]}
WIDE_BWD = {"float32": [("F32ELb0E.*Li128ELi128E", (71, 31), (33, 9))], "bfloat16": [("BF16ELb0E.*Li128ELi128E", (71, 61), (33, 17))],
            "float16": [("F16ELb0E.*Li128ELi128E", (71, 61), (33, 17))]}
WIDE_CALL = (700, 2, 2)  # T, k, E


@pytest.mark.parametrize("dtype,shape", [(t, s) for t in TYPES for s in WIDE[t]], ids=str)
@pytest.mark.parametrize("form", ["relu", "combine"])
def test_linear_of_wide_matrices(torch, isc, dtype, shape, form):
    """The tiles that no smaller call takes: fp32's of 128, those through registers, sums by all."""
    (T, k, E), (_, (K, _), (N, groups)), combine = WIDE_CALL, shape, form == "combine"
    rt, ids = route(torch, isc, 31, T, k, E, 0.05)
    x, w = operands(torch, 31, T, k, E, K, N, dtype, not combine, combine)
    got = isc.isc_expert_linear(x, w.repeat(1, groups, 1), rt, relu=not combine, combine=combine)
    want, size = train.expert_linear(host(x), host(w), ids, not combine, host(rt.weights) if combine else None)
    close(host(got[..., :N]), want, (K + 64 + k * combine + 8 * (dtype == "float32")) * E24 * size, dtype, "y")
    assert (got.unflatten(-1, (groups, N)) == got[..., None, :N]).all()
    if not combine:
        assert (got[rt.ids < 0] == 0).all()


@pytest.mark.parametrize("dtype,shape", [(t, s) for t in TYPES for s in WIDE_BWD[t]], ids=str)
@pytest.mark.parametrize("form", ["relu", "combine", "plain"])
def test_bwd_of_wide_matrices(torch, isc, dtype, shape, form):
    """As above: dx and dw by fp32's tiles of 128, and by those of rows that are off 16 bytes."""
    (T, k, E), (_, (K, many), (N, groups)), combine = WIDE_CALL, shape, form == "combine"
    rt, ids = route(torch, isc, 32, T, k, E, 0.05)
    x, w = operands(torch, 32, T, k, E, K, N, dtype, not combine, combine)
    dy = dev(torch, np.random.default_rng(33).standard_normal((T, N) if combine else (T, k, N)), dtype)
    dd = torch.cat([dy] + [torch.zeros_like(dy)] * (groups - 2) + [dy], -1)  # the first and the last group of outputs
    y = torch.relu(dev(torch, np.random.default_rng(34).standard_normal((T, k, N)), dtype)) if form == "relu" else None
    got = isc.isc_expert_linear_bwd(dd, x.repeat(*([1] * (x.dim() - 1)), many), w.repeat(1, groups, many), rt,
                                    y=None if y is None else y.repeat(1, 1, groups), combine=combine)
    want = train.expert_linear_bwd(host(dy), host(x), host(w), ids, None if y is None else host(y), host(rt.weights) if combine else None)
    parts = 8 * (dtype == "float32")
    value, size = want["dx"]
    dx = got.dx.unflatten(-1, (many, K))
    close(host(dx[..., 0, :]), 2 * value, (2 * N + 64 + k + parts) * E24 * 2 * size, dtype, "dx")
    assert (dx == dx[..., :1, :]).all()
    value, size = want["dw"]
    dw = got.dw.unflatten(-1, (many, K)).unflatten(1, (groups, N))
    close(host(dw[:, 0, :, 0]), value, ((T * k + 64 + parts) * E24 + (U[dtype] if combine else 0)) * size
          + (TINY * T * k * np.abs(host(x)).max() if combine and dtype == "float16" else 0), dtype, "dw")
    assert (dw[:, 0] == dw[:, 0, :, :1]).all() and (dw[:, -1] == dw[:, 0]).all() and (dw[:, 1:-1] == 0).all()
    if combine:
        value, size = want["dweights"]
        close(host(got.dweights), 2 * many * value, (2 * N + many * K + 64 + parts) * E24 * 2 * many * size, "float32", "dweights")


@pytest.mark.parametrize("shape", [(3, 130, 65), (1, 72, 465), (1, 465, 72), (2, 521, 301), (2, 301, 521), (1, 200, 328), (1, 130, 1100)], ids=str)
def test_orthogonalize_in_a_workspace_of_its_size(torch, isc, shape):
    """NaN in it and a guard behind its end: matrices by tiles, with sums in parts and without, wide and tall."""
    ws = nothing_in_it(torch, isc, "isc_orthogonalize_workspace_size", *shape)
    whole = torch.full((ws.numel() + 4096,), 255, dtype=torch.uint8, device="cuda")
    for dtype in TYPES:
        g = dev(torch, gradient(41, *shape, 3), dtype)
        whole.fill_(255)
        assert torch.equal(isc.isc_orthogonalize(g, ws=whole[:ws.numel()]), isc.isc_orthogonalize(g))
        assert (whole[ws.numel():] == 255).all()


@pytest.mark.parametrize("what", ["hole", "taken away", "another's"])
def test_lists_that_ids_do_not_agree_with_by_the_largest_tiles(torch, isc, what):
    """Rows, sums and dweights by tiles of 256 x 256 are those of lists made for the pairs that are left."""
    T, k, E, K, N, many = 700, 2, 2, 72, 40, 140
    rt, left = disturbed(torch, isc, what, 51, T, k, E)
    offsets, order = train.lists(left, E)
    clean = isc.Route(*(torch.from_numpy(np.ascontiguousarray(v)).cuda() for v in (left, host(rt.weights).astype(np.float32), offsets, order)))
    x, w = operands(torch, 51, T, k, E, K, N, "bfloat16", True)
    wide = w.repeat(1, many, 1)
    desc = isc.ExpertDesc(E, N * many, K, 2, k, 1)
    for combine in (False, True):
        ws = nothing_in_it(torch, isc, "isc_expert_linear_workspace_size", desc, T, combine)
        leave_nan(torch, x.new_empty((T, N * many) if combine else (T, k, N * many)))
        assert torch.equal(isc.isc_expert_linear(x, wide, rt, combine=combine, ws=ws),
                           isc.isc_expert_linear(x, wide, clean, combine=combine))
    wide = w.repeat(1, 1, many)
    for shared in (True, False):
        xx = (x if shared else x[:, None].expand(-1, k, -1)).repeat(*([1] * (1 if shared else 2)), many)
        desc = isc.ExpertDesc(E, N, K * many, 2, k, shared)
        dy = dev(torch, np.random.default_rng(52).standard_normal((T, N)), "bfloat16")
        ws = nothing_in_it(torch, isc, "isc_expert_linear_bwd_workspace_size", desc, T, 0, 1)
        leave_nan(torch, xx, rt.weights)
        got = isc.isc_expert_linear_bwd(dy, xx, wide, rt, combine=True, ws=ws)
        want = isc.isc_expert_linear_bwd(dy, xx, wide, clean, combine=True)
        assert torch.equal(got.dx, want.dx) and torch.equal(got.dweights, want.dweights)
