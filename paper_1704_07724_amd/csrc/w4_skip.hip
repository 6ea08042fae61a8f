// Products on 4-bit weights for a rectified x, its zeros skipped:
//   y[t][n] = sum over slots j of weight[t][j] * sum over k with x != 0 of w[n][k] x[t][j][k]
//
// The convolution's step on a matrix: inputs are tested 64 at a time by a
// ballot, and each nonzero reads one contiguous row of weights, lanes running
// over outputs.  The bytes moved are the nonzeros' rows and the scales of the
// groups of 32 inputs that hold one.  Products are summed per group in fp32 and
// then scaled, so a scale is applied once a group and not once a weight.
//
// The inputs (of all a token's slots) are cut into ranges, a workgroup each;
// its wavefronts take 64 inputs in turn.  Their sums meet in LDS in order, the
// ranges' in a second launch, so a result does not depend on timing.
#include "ffn.hpp"

namespace isc {
namespace {

using f32x2 = float __attribute__((ext_vector_type(2)));

constexpr int kWaves = 8;
constexpr int kOutputs = 512;  // outputs of a workgroup: eight a lane

__device__ __forceinline__ void add_row(float (&sum)[8], uint32_t w, float x) {
    f32x2 v;
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
    sum[0] = fmaf(v[0], x, sum[0]);
    sum[1] = fmaf(v[1], x, sum[1]);
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
    sum[2] = fmaf(v[0], x, sum[2]);
    sum[3] = fmaf(v[1], x, sum[3]);
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
    sum[4] = fmaf(v[0], x, sum[4]);
    sum[5] = fmaf(v[1], x, sum[5]);
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    sum[6] = fmaf(v[0], x, sum[6]);
    sum[7] = fmaf(v[1], x, sum[7]);
}

__global__ void __launch_bounds__(64 * kWaves) w4_skip_kernel(W4Args a, int ranges) {
    __shared__ float sums[kWaves][kOutputs];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t np = a.w.np();
    const int cols = static_cast<int>((np + kOutputs - 1) / kOutputs);
    const int64_t t = blockIdx.x / cols;
    const int c0 = static_cast<int>(blockIdx.x % cols) * kOutputs;
    const int n0 = c0 + lane * 8;
    const int range = blockIdx.y;
    const int slots = a.slots ? a.slots : 1;
    const int per = (a.w.K + 63) / 64;  // items of a slot
    const int64_t items = static_cast<int64_t>(per) * slots;
    const bool mine = n0 < np;
    float acc[8] = {};
    for (int64_t item = static_cast<int64_t>(range) * kWaves + wave; item < items;
         item += static_cast<int64_t>(ranges) * kWaves) {
        const int j = static_cast<int>(item / per), k0 = static_cast<int>(item % per) * 64;
        const int64_t row = t * slots + j;
        const uint8_t *w = a.packed;
        float factor = 1.0f;
        if (a.slots) {
            const int e = a.ids[row];
            if (e < 0 || e >= a.w.E) continue;
            factor = a.weights[row];
            w += static_cast<int64_t>(e) * a.w.row_bytes();
        }
        const int k = k0 + lane;
        const float x = k < a.w.K ? load_as(a.x, row * a.ldx + k, a.xtype) : 0.0f;
        const unsigned long long nz = __ballot(x != 0.0f);
        for (int half = 0; half < 2; ++half) {
            uint32_t m = static_cast<uint32_t>(nz >> (32 * half));
            if (m == 0u) continue;
            const uint8_t *base = w + (k0 / 32 + half) * 17 * np;
            uint2 sc = make_uint2(0u, 0u);
            if (mine) sc = *reinterpret_cast<const uint2 *>(base + n0);
            float sum[8] = {};
            while (m) {
                const int i = __builtin_ctz(m);
                m &= m - 1;
                const float xv = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 32 * half + i));
                uint32_t q = 0u;
                if (mine) q = *reinterpret_cast<const uint32_t *>(base + np + i * (np / 2) + n0 / 2);
                add_row(sum, q, xv);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                acc[i] = fmaf(sum[i] * factor, scale_value(((i < 4 ? sc.x : sc.y) >> (8 * (i & 3))) & 255u), acc[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wave][lane * 8 + i] = acc[i];
    __syncthreads();
    const int64_t n = c0 + static_cast<int>(threadIdx.x);
    float v = 0.0f;
#pragma unroll
    for (int z = 0; z < kWaves; ++z) v += sums[z][threadIdx.x];
    if (n >= a.w.N) return;
    if (ranges == 1)
        store_as(a.y, t * a.ldy + n, v, a.ytype);
    else
        a.part[(static_cast<int64_t>(range) * a.T + t) * a.w.N + n] = v;
}

__global__ void __launch_bounds__(256) w4_ranges_kernel(W4Args a, int ranges) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t all = static_cast<int64_t>(a.T) * a.w.N;
    if (i >= all) return;
    float v = 0.0f;
    for (int r = 0; r < ranges; ++r) v += a.part[r * all + i];
    store_as(a.y, i / a.w.N * a.ldy + i % a.w.N, v, a.ytype);
}

}  // namespace

int w4_skip_ranges(const W4Shape &w, int T, int slots) {
    const int64_t items = (w.K + 63) / 64 * static_cast<int64_t>(slots ? slots : 1);
    const int64_t cols = (w.np() + kOutputs - 1) / kOutputs;
    int64_t ranges = 2048 / (cols * (T > 0 ? T : 1));
    const int64_t most = (items + kWaves - 1) / kWaves;
    if (ranges > most) ranges = most;
    if (ranges > 64) ranges = 64;
    return ranges < 1 ? 1 : static_cast<int>(ranges);
}

hipError_t launch_w4_skip(const W4Args &a, hipStream_t s) {
    const int ranges = w4_skip_ranges(a.w, a.T, a.slots);
    const dim3 grid(static_cast<unsigned>((a.w.np() + kOutputs - 1) / kOutputs * a.T), static_cast<unsigned>(ranges));
    w4_skip_kernel<<<grid, dim3(64 * kWaves), 0, s>>>(a, ranges);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || ranges == 1) return e;
    const int64_t all = static_cast<int64_t>(a.T) * a.w.N;
    w4_ranges_kernel<<<dim3(static_cast<unsigned>((all + 255) / 256)), dim3(256), 0, s>>>(a, ranges);
    return hipGetLastError();
}

}  // namespace isc
