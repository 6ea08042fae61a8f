"""What the feed-forward operators launch, on the host: the library runs over a
recorder in place of the HIP runtime, which notes every kernel with its grid and
runs nothing.  So calls can be looked at that are too large to make here, and calls
that have no addresses to read."""
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
A, B, C, D, E, F, G = (0x4000000000000 * i for i in range(1, 8))  # addresses that are only compared

RECORDER = r"""
#include <hip/hip_runtime_api.h>
#include <cstdio>
#include <cstring>
#include <map>
#include <string>

namespace {
std::map<const void *, std::string> names;
std::string log;
struct Call { dim3 grid, block; size_t lds; hipStream_t stream; } call;
}  // namespace

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *handle; return &handle; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, dim3 *, dim3 *,
                           int *) { names[host] = name; }
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, hipStream_t s) { call = Call{g, b, lds, s}; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *lds, hipStream_t *s) {
    *g = call.grid; *b = call.block; *lds = call.lds; *s = call.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 g, dim3 b, void **, size_t lds, hipStream_t) {
    char dims[200];
    std::snprintf(dims, sizeof dims, " %u %u %u %u %u %u %zu\n", g.x, g.y, g.z, b.x, b.y, b.z, lds);
    log += names[f] + dims;
    return hipSuccess;
}
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipGetDevicePropertiesR0600(hipDeviceProp_tR0600 *p, int) {
    std::memset(p, 0, sizeof *p);
    std::strcpy(p->gcnArchName, "gfx950");
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipFuncSetAttribute(const void *, hipFuncAttribute, int) { return hipSuccess; }
const char *recorded() { static std::string s; s = log; log.clear(); return s.c_str(); }
}
"""

RUN = r"""
import ctypes, json, sys
recorder = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)  # found before the runtime that the library names
recorder.recorded.restype = ctypes.c_char_p
import paper_1704_07724_amd as isc
out = []
for name, args in json.loads(sys.stdin.read()):
    args = [isc.W4Desc(*a) if isinstance(a, list) else a for a in args]
    n = ctypes.c_size_t()
    status = getattr(isc.lib(), name)(*args, *([n] if name.endswith("_size") else []))
    kernels = [line.split() for line in recorder.recorded().decode().splitlines()]
    out.append((status, n.value, [(k[0], [int(v) for v in k[1:]]) for k in kernels]))
print(json.dumps(out))
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """launches([(entry point, arguments), ...]) -> [(status, size, [(kernel, [grid, block, bytes of LDS]), ...]), ...]"""
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


def norm_bwd(T, N, t=2, **kw):
    a = dict(dy=A, h=B, w=C, rstd=D, dh=None, dx=E, dw=F, ws=G)
    a.update(kw)
    return "isc_rmsnorm_bwd", [T, N, t, a["dy"], N, a["h"], N, a["w"], t, a["rstd"], a["dh"], N, a["dx"], N, a["dw"],
                               a["ws"], 1 << 40, None]


def test_norm_bwd_without_rows(launches):
    """No kernel that reads a row or the weight: the sums of nothing alone are written."""
    none = dict(dy=None, h=None, w=None, rstd=None, dx=None)
    shapes = [(N, t) for N in (1, 64, 512, 1000, 4096, 16384) for t in (0, 1, 2)]
    for (N, t), (status, _, kernels) in zip(shapes, launches([norm_bwd(0, N, t, **none) for N, t in shapes])):
        assert status == 0 and len(kernels) == 1 and "column_sum" in kernels[0][0], (N, t, kernels)
        assert kernels[0][1][0] == (N + 31) // 32
    (_, _, kernels), = launches([norm_bwd(1, 64)])
    assert len(kernels) == 2 and "rmsnorm_bwd" in kernels[0][0]


def norm(T, N, t=2):
    return "isc_rmsnorm", [T, N, t, A, N, B, N, C, t, 1e-6, D, N, E, N, F, N, G, (N + 31) // 32, None, None]


def launchable(kernels):
    """Every grid is one that a launch takes, with a workgroup at least; returns the kernels' workgroups."""
    for name, (x, y, z, bx, by, bz, lds) in kernels:
        assert 0 < x * bx < 2 ** 32 and 0 < y <= 65535 and z == by == bz == 1 and 0 < bx <= 1024 and lds <= 65536, \
            (name, x, y, bx, lds)
    return [k[1][0] for k in kernels]


def test_norm_of_many_rows(launches):
    """A workgroup a row, in as many launches as it takes."""
    shapes = [(T, N, t) for T in (1, 2 ** 22 - 1, 2 ** 22, 2 ** 22 + 1, 2 ** 26, 2 ** 26 + 5, 2 ** 31 - 1)
              for N in (1, 64, 512, 513, 4096, 8192, 65536) for t in (0, 1, 2)]
    for (T, N, t), (status, _, kernels) in zip(shapes, launches([norm(*s) for s in shapes])):
        assert status == 0 and sum(launchable(kernels)) == T, (T, N, t)


def test_norm_bwd_of_many_rows(launches):
    """The count of workgroups holds up to the largest count of rows, and the workspace with it."""
    shapes = [(T, N) for T in (2 ** 22, 2 ** 31 - 8, 2 ** 31 - 1) for N in (1, 64, 512, 513, 4096, 16384)]
    calls = [norm_bwd(*s) for s in shapes] + [("isc_rmsnorm_bwd_workspace_size", list(s)) for s in shapes]
    out = launches(calls)
    for (T, N), (status, _, kernels), (_, size, _) in zip(shapes, out, out[len(shapes):]):
        assert status == 0 and launchable(kernels)[0] >= 256 and size == 4 * N * kernels[0][1][0], (T, N, kernels)


def route_bwd(T, N, k):
    return "isc_route_bwd", [T, N, k, 2, A, B, N, C, 0, 1, 1.0, D, N, None]


def test_route_bwd_of_many_tokens(launches):
    """Four tokens a workgroup, in as many launches as it takes."""
    shapes = [(T, N) for T in (1, 2 ** 26 - 5, 2 ** 26 - 4, 2 ** 26 - 3, 2 ** 26, 2 ** 30 + 1, 2 ** 31 - 1) for N in (2, 64, 1024)]
    for (T, N), (status, _, kernels) in zip(shapes, launches([route_bwd(*s, 2) for s in shapes])):
        assert status == 0 and sum(launchable(kernels)) == (T + 3) // 4, (T, N, kernels)


def route(T, N, k, groups=1):
    return "isc_route", [T, N, k, 2, A, N, None, 1, groups, groups, 1, 1.0, B, C, D, E, F, 1 << 50, None]


def test_route_of_many_tokens(launches):
    """Up to the limit on tokens every launch is one that the device takes; past it the call and the
    workspace's size are refused, not the launch."""
    most = 2 ** 28 - 64
    for N, k, groups in ((2, 1, 1), (64, 7, 1), (100, 7, 2), (300, 5, 4), (600, 3, 1)):
        sizes = [("isc_route_workspace_size", [T, N]) for T in (most, most + 1, 2 ** 31 - 1)]
        out = launches([route(T, N, k, groups) for T in (2 ** 22, most, most + 1, 2 ** 31 // k - 1)] + sizes)
        for status, _, kernels in out[:2]:
            assert status == 0 and len(kernels) == 2 and launchable(kernels), (N, kernels)
        assert [(o[0], o[2]) for o in out[2:4]] == [(3, []), (3, [])], out[2:4]
        assert [o[0] for o in out[4:]] == [0, 3, 3]


def skip(T, N, K, slots=0, E_=1):
    return "isc_w4_skip", [[E_, N, K, 1], A, T, B, 2, K, slots, C if slots else None, D if slots else None, E, 2, N, F, 1 << 50,
                           None]


def test_skip_of_many_tokens(launches):
    """512 outputs of a token a workgroup, in as many launches as it takes."""
    shapes = [(T, N, slots) for T in (1, 2 ** 19 - 1, 2 ** 19, 2 ** 20) for N in (1, 4096, 4097, 8192, 2 ** 24) for slots in (0, 3)]
    for (T, N, slots), (status, _, kernels) in zip(shapes, launches([skip(T, N, 256, slots, 2 if slots else 1)
                                                                     for T, N, slots in shapes])):
        assert status == 0 and launchable(kernels), (T, N)
        across = -(-(-(-N // 128) * 128) // 512)
        assert sum(k[1][0] for k in kernels if "w4_skip" in k[0]) == T * across, (T, N, slots)


def linear(T, N, K, xt, slots=0, E_=1):
    per = (B, None) if xt != 3 else (B, C)
    return "isc_w4_linear", [[E_, N, K, 0], A, T, per[0], xt, K, per[1], (K + 31) // 32, slots, C + (1 << 48) if slots else None,
                             C + (1 << 49) if slots else None, D if slots else None, E, 2, N, 0, F, 1 << 55, None]


def test_linear_of_many_tokens(launches):
    """Up to the limits on tokens and inputs x is laid out and multiplied by launches that the device takes."""
    shapes = [(T, N, K, xt) for T in (1, 17, 2 ** 17, 2 ** 20) for N, K in ((16, 8), (48, 8), (48, 16384), (16, 65536), (4096, 32768),
                                                                         (16, 2 ** 24), (2 ** 24, 16)) for xt in (0, 1, 2, 3)]
    calls = [linear(*s) for s in shapes]
    sizes = [("isc_w4_linear_workspace_size", [[1, N, K, 0], T, xt, 0]) for T, N, K, xt in shapes]
    out = launches(calls + sizes)
    for shape, (status, _, kernels), (st, size, _) in zip(shapes, out, out[len(shapes):]):
        assert st == 0 and (size == 0 or size >= shape[0] * shape[2] * 2), shape
        assert status == 0 and launchable(kernels) and "w4_linear" in kernels[-1][0], (shape, kernels)


def test_linear_of_many_tokens_by_experts(launches):
    shapes = [(T, N, K, xt) for T in (1, 2 ** 20) for N, K in ((16, 8), (4096, 4096), (2 ** 20, 32)) for xt in (0, 1, 2, 3)]
    for shape, (status, _, kernels) in zip(shapes, launches([linear(*s, slots=4, E_=1024) for s in shapes])):
        assert status == 0 and launchable(kernels), (shape, kernels)


def test_weights_of_any_size(launches):
    """Quantising and laying out up to the limits on a matrix and on their count."""
    descs = [[e, n, k, layout] for e in (1, 1024) for n, k in ((1, 1), (2 ** 24, 1), (2 ** 24, 3000), (3000, 2 ** 24), (2 ** 18, 2 ** 17))
             for layout in (0, 1)]
    calls = [("isc_w4_quantize", [d, A, 2, d[2], D, F, None]) for d in descs]
    calls += [("isc_w4_pack_codes", [d, A, D, F, None]) for d in descs]
    for (name, args), (status, _, kernels) in zip(calls, launches(calls)):
        assert status == 0 and launchable(kernels), (name, args, kernels)
