"""The refusals of the operators that train a routed block, on the host, and what
they launch: the C entry points turn bad arguments into a status before they touch
a device; over a recorder in place of the HIP runtime every grid is one that a
launch takes, up to the limits."""
import ctypes
import json
import os
import re
import subprocess
import sys

import pytest

import paper_1704_07724_amd as isc
import test_gpu_train as wide
from test_ffn_launches import RECORDER, ROCM, ROOT

NULL, SHAPE, LIMIT, WORKSPACE, ALIAS, DEVICE, ALIGN, ARG = 1, 2, 3, 4, 5, 7, 9, 10
OK = (0, DEVICE)  # valid arguments: with no GPU in the process the device check ends the call
W, X, Y, DY, IDS, WT, OFF, ORD, DX, DW, DS, WS = (0x10000000 * i for i in range(1, 13))  # addresses that are only compared


@pytest.fixture(scope="module", autouse=True)
def no_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("made-up addresses: only where no call can reach a GPU")


def desc(E=4, N=24, K=40, t=2, slots=2, shared=1):
    return isc.ExpertDesc(E, N, K, t, slots, shared)


def linear(d=None, w=W, ldw=40, T=3, x=X, ldx=40, ids=IDS, wt=None, off=OFF, order=ORD, y=Y, yt=2, ldy=24, relu=1, combine=0,
           ws=WS, n=1 << 24):
    return isc.lib().isc_expert_linear(d or desc(), w, ldw, T, x, ldx, ids, wt, off, order, y, yt, ldy, relu, combine, ws, n, None)


def test_linear_refusals():
    assert linear() in OK and linear(relu=0) in OK and linear(relu=0, combine=1, wt=WT) in OK and linear(yt=0) in OK
    assert linear(T=0, x=None, y=None, ids=None, off=None, order=None, ws=None) == 0
    for name in ("w", "x", "ids", "off", "order", "y", "ws"):
        assert linear(**{name: None}) == NULL, name
    assert linear(relu=0, combine=1) == NULL  # no weights
    assert isc.lib().isc_expert_linear(None, W, 40, 3, X, 40, IDS, None, OFF, ORD, Y, 2, 24, 0, 0, WS, 1 << 20, None) == NULL
    assert linear(relu=1, combine=1, wt=WT) == ARG and linear(yt=3) == ARG and linear(desc(t=3)) == ARG
    for bad in (dict(E=0), dict(N=0), dict(K=0), dict(slots=0)):
        assert linear(desc(**bad)) == SHAPE, bad
    assert linear(T=-1) == SHAPE and linear(ldx=39) == SHAPE and linear(ldw=39) == SHAPE and linear(ldy=23) == SHAPE
    assert linear(desc(E=1025)) == LIMIT and linear(desc(slots=65)) == LIMIT and linear(T=2 ** 20 + 1) == LIMIT
    assert linear(desc(K=2 ** 20 + 1), ldw=2 ** 21, ldx=2 ** 21) == LIMIT and linear(desc(N=2 ** 20 + 1), ldy=2 ** 21) == LIMIT
    assert linear(desc(N=2 ** 20, slots=64), T=2 ** 20, ldy=2 ** 20, n=1 << 60) == LIMIT  # more tiles than are counted
    assert linear(x=X + 1) == ALIGN and linear(w=W + 1) == ALIGN and linear(y=Y + 1) == ALIGN and linear(ids=IDS + 2) == ALIGN
    assert linear(off=OFF + 1) == ALIGN and linear(order=ORD + 2) == ALIGN and linear(ws=WS + 16) == ALIGN
    assert linear(yt=0, y=Y + 2) == ALIGN and linear(x=X + 2) in OK
    for at in (W, X, IDS, OFF, ORD, WS):
        assert linear(y=at) == ALIAS, at
    assert linear(ws=X) == ALIAS and linear(relu=0, combine=1, wt=WT, y=WT) == ALIAS
    n = ctypes.c_size_t()
    assert isc.lib().isc_expert_linear_workspace_size(desc(), 3, 0, None) == NULL
    assert isc.lib().isc_expert_linear_workspace_size(desc(), 3, 0, n) == 0 and n.value > 0
    assert linear(n=n.value) in OK and linear(n=n.value - 1) == WORKSPACE
    lone = n.value
    assert isc.lib().isc_expert_linear_workspace_size(desc(), 3, 1, n) == 0 and n.value >= lone + 6 * 24 * 4


def bwd(d=None, w=W, ldw=40, T=3, x=X, ldx=40, dy=DY, lddy=24, y=Y, ldy=24, ids=IDS, wt=None, off=OFF, order=ORD, combine=0, dx=DX,
        lddx=40, dw=DW, ds=None, ws=WS, n=1 << 24):
    return isc.lib().isc_expert_linear_bwd(d or desc(), w, ldw, T, x, ldx, dy, lddy, y, ldy, ids, wt, off, order, combine, dx, lddx, dw,
                                           ds, ws, n, None)


def test_bwd_refusals():
    assert bwd() in OK and bwd(y=None) in OK and bwd(dx=None) in OK and bwd(dw=None) in OK
    assert bwd(y=None, combine=1, wt=WT, ds=DS) in OK and bwd(y=None, combine=1, wt=WT, dx=None, dw=None, ds=DS) in OK
    for name in ("w", "x", "dy", "ids", "off", "order", "ws"):
        assert bwd(**{name: None}) == NULL, name
    assert bwd(dx=None, dw=None) == NULL and bwd(y=None, combine=1) == NULL
    nothing = dict(w=None, x=None, dy=None, y=None, ids=None, off=None, order=None, ws=None, n=0)
    assert bwd(T=0, **nothing) in OK       # dw = 0 is still written
    assert bwd(T=0, dw=None, **nothing) == 0
    assert bwd(ds=DS) == ARG and bwd(combine=1, wt=WT) == ARG  # weights' gradient without a sum; a sum with a rectified output
    assert bwd(T=-1) == SHAPE and bwd(lddy=23) == SHAPE and bwd(ldy=23) == SHAPE and bwd(lddx=39) == SHAPE and bwd(ldx=1) == SHAPE
    assert bwd(desc(t=5)) == ARG and bwd(desc(E=2000)) == LIMIT
    for name in ("w", "x", "dy", "y", "dx", "dw"):
        assert bwd(**{name: dict(w=W, x=X, dy=DY, y=Y, dx=DX, dw=DW)[name] + 1}) == ALIGN, name
    assert bwd(ws=WS + 128) == ALIGN and bwd(y=None, combine=1, wt=WT, ds=DS + 2) == ALIGN
    for at in (W, X, DY, Y, IDS, ORD):
        assert bwd(dx=at) == ALIAS and bwd(dw=at) == ALIAS, at
    assert bwd(dx=DW) == ALIAS and bwd(ws=DX) == ALIAS and bwd(y=None, combine=1, wt=WT, ds=DX) == ALIAS
    n = ctypes.c_size_t()
    assert isc.lib().isc_expert_linear_bwd_workspace_size(desc(), 3, 1, 0, n) == 0
    assert bwd(n=n.value) in OK and bwd(n=n.value - 1) == WORKSPACE
    assert isc.lib().isc_expert_linear_bwd_workspace_size(desc(), 3, 1, 1, n) == ARG


def orth(B=2, M=24, N=40, t=2, g=X, ldg=40, steps=2, coef=(3.4445, -4.775, 2.0315) * 2, eps=1e-7, o=Y, ot=2, ldo=40, ws=WS, n=1 << 24):
    c = None if coef is None else (ctypes.c_float * len(coef))(*coef)
    return isc.lib().isc_orthogonalize(B, M, N, t, g, ldg, steps, c, eps, o, ot, ldo, ws, n, None)


def test_orthogonalize_refusals():
    assert orth() in OK and orth(t=0) in OK and orth(ot=1) in OK and orth(B=0, g=None, o=None, ws=None) == 0
    assert orth(g=None) == NULL and orth(o=None) == NULL and orth(ws=None) == NULL and orth(coef=None) == NULL
    assert orth(M=0) == SHAPE and orth(N=0) == SHAPE and orth(B=-1) == SHAPE and orth(ldg=39) == SHAPE and orth(ldo=39) == SHAPE
    assert orth(M=65537) == LIMIT and orth(N=65537, ldg=70000, ldo=70000) == LIMIT and orth(B=65536) == LIMIT
    assert orth(t=3) == ARG and orth(ot=0) == ARG and orth(ot=3) == ARG and orth(steps=0) == ARG and orth(steps=65) == ARG
    assert orth(eps=-1.0) == ARG and orth(eps=float("nan")) == ARG and orth(eps=float("inf")) == ARG
    # values that a polynomial takes out of range, at an end and in between, at once and by steps
    assert orth(coef=(16.0, 0, 0) * 1 + (1.0, 0, 0)) in OK and orth(coef=(16.1, 0, 0) + (1.0, 0, 0)) == ARG
    assert orth(coef=(4.1, 0, 0) * 2) == ARG and orth(coef=(60.0, -60.0, 0.0) + (0.1, 0, 0)) == ARG
    assert orth(coef=(0.0, 0.0, 600.0) + (0.0, 0, 0)) == ARG and orth(coef=(float("nan"), 0, 0) * 2) == ARG
    assert orth(coef=(1.0, float("inf"), 0) * 2) == ARG
    assert orth(g=X + 1) == ALIGN and orth(o=Y + 1) == ALIGN and orth(ws=WS + 8) == ALIGN and orth(t=0, g=X + 2) == ALIGN
    assert orth(o=X) in OK and orth(o=X + 80) == ALIAS and orth(ws=X) == ALIAS and orth(ws=Y) == ALIAS and orth(t=0, o=X) == ALIAS
    n = ctypes.c_size_t()
    assert isc.lib().isc_orthogonalize_workspace_size(2, 24, 40, n) == 0
    assert orth(n=n.value) in OK and orth(n=n.value - 1) == WORKSPACE
    assert isc.lib().isc_orthogonalize_workspace_size(2, 24, 40, None) == NULL


RUN = r"""
import ctypes, json, sys
recorder = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)  # found before the runtime that the library names
recorder.recorded.restype = ctypes.c_char_p
import paper_1704_07724_amd as isc
out = []
for name, args in json.loads(sys.stdin.read()):
    args = [(isc.ExpertDesc if len(a) == 6 and all(isinstance(v, int) for v in a) else (ctypes.c_float * len(a)))(*a)
            if isinstance(a, list) else a for a in args]
    n = ctypes.c_size_t()
    status = getattr(isc.lib(), name)(*args, *([n] if name.endswith("_size") else []))
    kernels = [line.split() for line in recorder.recorded().decode().splitlines()]
    out.append((status, n.value, [(k[0], [int(v) for v in k[1:]]) for k in kernels]))
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("recorder")
    src, so = tmp / "recorder.cpp", tmp / "recorder.so"
    src.write_text(RECORDER)
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-w", "-D__HIP_PLATFORM_AMD__=1", "-I", os.path.join(ROCM, "include"),
                    str(src), "-o", str(so)], check=True)

    def run(calls):
        r = subprocess.run([sys.executable, "-c", RUN, str(so)], input=json.dumps(calls), cwd=ROOT, capture_output=True,
                           text=True, timeout=300)
        assert r.returncode == 0, r.stderr
        return json.loads(r.stdout.splitlines()[-1])
    return run


FAR = [i << 56 for i in range(1, 100)]  # so far apart that no tensor reaches the next


def launchable(kernels):
    for name, (x, y, z, bx, by, bz, lds) in kernels:
        assert 0 < x * bx < 2 ** 32 and 0 < y <= 65535 and z == by == bz == 1 and 0 < bx <= 1024 and lds <= 163840, (name, x, y, bx, lds)
    return kernels


SIZES = [(1, 1, 1, 1, 1), (1, 64, 8, 2048, 1408), (16, 64, 8, 2048, 1408), (4096, 64, 8, 2048, 1408), (2 ** 20, 1, 1, 64, 64),
         (2 ** 20, 1024, 64, 64, 64), (5, 1024, 64, 16, 2 ** 20), (2 ** 20, 8, 2, 4096, 16384), (300, 3, 2, 2 ** 20, 40)]


def test_linear_launches(launches):
    shapes = [(s, t, c) for s in SIZES for t in (0, 1, 2) for c in (0, 1)]
    a = FAR
    calls = [("isc_expert_linear", [[E, N, K, t, k, 1], a[0], K, T, a[1], K, a[2], a[3], a[4], a[5], a[6], t, N, 0, c, a[7], 1 << 55, None])
             for (T, E, k, K, N), t, c in shapes]
    sizes = [("isc_expert_linear_workspace_size", [[E, N, K, t, k, 1], T, c]) for (T, E, k, K, N), t, c in shapes]
    out = launches(calls + sizes)
    for shape, (status, _, kernels), (st, size, _) in zip(shapes, out, out[len(shapes):]):
        (T, E, k, K, N), t, c = shape
        assert status == st == 0 and launchable(kernels), (shape, status, st)
        few = T * k <= (8 if t == 0 else 4) * E
        assert len(kernels) == (1 if few else 2) + c, (shape, kernels)
        assert size >= T * k * N * 4 * c


def test_bwd_launches(launches):
    shapes = [(s, t, f) for s in SIZES for t in (0, 1, 2) for f in ("relu", "combine", "plain")]
    a = FAR
    calls = [("isc_expert_linear_bwd", [[E, N, K, t, k, 1], a[0], K, T, a[1], K, a[2], N, a[3] if f == "relu" else None, N, a[4], a[5],
                                        a[6], a[7], int(f == "combine"), a[8], K, a[9], a[10] if f == "combine" else None, a[11],
                                        1 << 55, None]) for (T, E, k, K, N), t, f in shapes]
    sizes = [("isc_expert_linear_bwd_workspace_size", [[E, N, K, t, k, 1], T, int(f == "relu"), int(f == "combine")])
             for (T, E, k, K, N), t, f in shapes]
    out = launches(calls + sizes)
    for shape, (status, _, kernels), (st, size, _) in zip(shapes, out, out[len(shapes):]):
        (T, E, k, K, N), t, f = shape
        assert status == st == 0 and launchable(kernels), (shape, status, st)
        # the plan, masked or weighted gradients, dx, its sum over slots, dweights, dw
        assert len(kernels) == 3 + (f != "plain") + (k > 1) + (f == "combine"), (shape, kernels)
        assert size >= (T * k * N * (4 if t == 0 else 2) if f != "plain" else 0) + (T * k * K * 4 if k > 1 else 0)


def test_no_tokens_launch_one_kernel_for_the_weights(launches):
    a = FAR
    (status, _, kernels), = launches([("isc_expert_linear_bwd", [[1024, 4096, 16384, 2, 2, 1], None, 16384, 0, None, 16384, None, 4096,
                                                                None, 4096, None, None, None, None, 0, a[0], 16384, a[1], None, None, 0,
                                                                None])])
    assert status == 0 and len(launchable(kernels)) == 1 and "zero" in kernels[0][0]


def test_orthogonalize_launches(launches):
    shapes = [(B, M, N) for B in (1, 3, 64) for M, N in ((1, 1), (64, 2048), (2048, 64), (777, 1155), (1408, 2048), (4096, 9216), (9216, 4096))]
    shapes += [(1, 65536, 65536), (65535, 8, 8), (1, 16, 65536), (1, 65536, 16), (1, 100, 4096)]
    a = FAR
    calls = [("isc_orthogonalize", [B, M, N, 0, a[0], N, 3, [1.5, -0.5, 0.0] * 3, 1e-7, a[1], 2, N, a[2], 1 << 55, None]) for B, M, N in shapes]
    for shape, (status, _, kernels) in zip(shapes, launches(calls)):
        assert status == 0 and launchable(kernels), shape
        # two launches and three a step, a fourth where A comes in parts; one a step where a side is at most 64
        assert len(kernels) in ((5,) if min(shape[1:]) <= 64 else (11, 14)), (shape, len(kernels))


def test_orthogonalize_stops_at_what_is_counted(launches):
    a = FAR
    (status, _, kernels), (size, _, _) = launches([
        ("isc_orthogonalize", [65535, 65536, 65536, 0, a[0], 65536, 1, [1.5, -0.5, 0.0], 1e-7, a[1], 2, 65536, a[2], 1 << 60, None]),
        ("isc_orthogonalize_workspace_size", [65535, 65536, 65536])])
    assert status == size == LIMIT and kernels == []


def test_an_empty_stack_of_any_shape(launches):
    """Nothing is launched and nothing divided by its number, also where A's sums would come in parts."""
    a = FAR
    shapes = [(1, 1), (24, 40), (128, 1024), (1024, 128), (65, 449), (777, 1155), (4096, 9216), (65536, 65536)]
    calls = [("isc_orthogonalize", [0, M, N, 0, a[0], N, 3, [1.5, -0.5, 0.0] * 3, 1e-7, a[1], 2, N, a[2], 1 << 55, None]) for M, N in shapes]
    sizes = [("isc_orthogonalize_workspace_size", [0, M, N]) for M, N in shapes]
    for shape, (status, _, kernels) in zip(shapes * 2, launches(calls + sizes)):
        assert status == 0 and kernels == [], shape


def test_the_wide_calls_take_the_tiles_that_they_are_for(launches):
    """By the names of the kernels that the GPU's tests of wide matrices launch."""
    (T, k, E), a, code = wide.WIDE_CALL, FAR, {"float32": 0, "float16": 1, "bfloat16": 2}
    forward, backward = ([(t, *s) for t in wide.TYPES for s in table[t]] for table in (wide.WIDE, wide.WIDE_BWD))
    calls = []
    for t, _, (K, _), (N, groups) in forward:
        for combine in (0, 1):
            calls.append(("isc_expert_linear", [[E, N * groups, K, code[t], k, 1 - combine], a[0], K, T, a[1], K, a[2], a[3], a[4], a[5],
                                                a[6], code[t], N * groups, 1 - combine, combine, a[7], 1 << 55, None]))
    for t, _, (K, many), (N, groups) in backward:
        for form in ("relu", "combine", "plain"):
            calls.append(("isc_expert_linear_bwd", [[E, N * groups, K * many, code[t], k, int(form != "combine")], a[0], K * many, T, a[1],
                                                    K * many, a[2], N * groups, a[3] if form == "relu" else None, N * groups, a[4], a[5],
                                                    a[6], a[7], int(form == "combine"), a[8], K * many, a[9],
                                                    a[10] if form == "combine" else None, a[11], 1 << 55, None]))
    expected = [pattern for _, pattern, _, _ in forward for _ in range(2)] + [pattern for _, pattern, _, _ in backward for _ in range(3)]
    for pattern, (status, _, kernels) in zip(expected, launches(calls)):
        names = [name for name, _ in kernels if "expert_rows" in name or "expert_dw" in name]
        assert status == 0 and names and all(re.search(pattern, name) for name in names), (pattern, names)


def test_coefficients_whose_largest_value_lies_between():
    """30 s - 30 s^3 has 11.5 at s^2 = 1/3 whatever little c s^5 is added: twice that is out of range."""
    for c in (0.0, 1e-20, -1e-20, 1e-12, -1e-12, 1e-6, -1e-6, 1e-3):
        assert orth(coef=(30.0, -30.0, c) + (1.3, 0, 0)) in OK and orth(coef=(30.0, -30.0, c) + (2.0, 0, 0)) == ARG, c
        assert orth(coef=(-30.0, 30.0, c) + (1.3, 0, 0)) in OK and orth(coef=(-30.0, 30.0, c) + (2.0, 0, 0)) == ARG, c
    # s - s^5 has 0.535 at s^4 = 1/5; 30 times that is in range, 31 is not
    assert orth(coef=(1.0, 0.0, -1.0) + (29.9, 0, 0)) in OK and orth(coef=(1.0, 0.0, -1.0) + (30.0, 0, 0)) == ARG
