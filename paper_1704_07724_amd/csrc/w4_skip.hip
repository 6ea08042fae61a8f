// Products on 4-bit weights for a rectified x, its zeros skipped:
//   y[t][n] = sum over slots j of weight[t][j] * sum over k with x != 0 of w[n][k] x[t][j][k]
//
// The convolution's step on a matrix: a wavefront tests 64 inputs or more by
// ballots and lists the nonzeros in LDS, then reads one contiguous row of weights for
// each, eight rows in flight, lanes running over outputs.  The bytes moved are
// the nonzeros' rows and the scales of the groups of 32 inputs that hold one.
// Products are summed per group in fp32 and then scaled, so a scale is applied
// once a group and not once a weight.
//
// The inputs (of all a token's slots) are cut into ranges, a workgroup each;
// its wavefronts take 64 TESTS inputs in turn.  Their sums meet in LDS in order, the
// ranges' in a second launch, so a result does not depend on timing.
//
// A chain of waits bounds it (the inputs, the rows, the sums, the second launch):
// 8192 outputs of 32768 inputs, a twentieth nonzero, one token, take 12.2 us for
// 13.6 MB (10.3 us on the GPU alone, 8 of them this kernel's), and 8 tokens of 8
// experts, 2048 outputs of 1408 with a tenth nonzero, 13.0 us for 13 MB.
#include "ffn.hpp"

namespace isc {
namespace {

using f32x2 = float __attribute__((ext_vector_type(2)));

constexpr int kWaves = 8;
constexpr int kOutputs = 512;  // outputs of a workgroup: eight a lane
constexpr int kFlight = 8;     // rows in flight

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

// A nonzero: its value and its place, the group's number times 32 and the
// input within it.
struct Entry {
    float x;
    int k;
};

template <int TESTS>
__global__ void __launch_bounds__(64 * kWaves) w4_skip_kernel(W4Args a, int ranges) {
    __shared__ Entry lists[kWaves][TESTS * 64 + kFlight];
    __shared__ float sums[kWaves][kOutputs];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t np = a.w.np();
    const int cols = static_cast<int>((np + kOutputs - 1) / kOutputs);
    const int64_t t = blockIdx.x / cols;
    const int c0 = static_cast<int>(blockIdx.x % cols) * kOutputs;
    const int range = blockIdx.y;
    const int slots = a.slots ? a.slots : 1;
    const int per = (a.w.K + TESTS * 64 - 1) / (TESTS * 64);  // turns of a slot
    const int64_t turns = static_cast<int64_t>(per) * slots;
    // lanes past the matrix's last outputs read its last ones again, for nothing
    const int64_t n0 = c0 + lane * 8 < np ? c0 + lane * 8 : np - 8;
    Entry *list = lists[wave];
    float acc[8] = {};
    for (int64_t turn = static_cast<int64_t>(range) * kWaves + wave; turn < turns;
         turn += static_cast<int64_t>(ranges) * kWaves) {
        const int j = static_cast<int>(turn / per), k0 = static_cast<int>(turn % per) * (TESTS * 64);
        const int64_t row = t * slots + j;
        const uint8_t *w = a.packed;
        float factor = 1.0f;
        if (a.slots) {
            const int e = a.ids[row];
            if (e < 0 || e >= a.w.E) continue;
            factor = a.weights[row];
            w += static_cast<int64_t>(e) * a.w.row_bytes();
        }
        float x[TESTS];
#pragma unroll
        for (int i = 0; i < TESTS; ++i) {
            const int k = k0 + i * 64 + lane;
            x[i] = k < a.w.K ? load_as(a.x, row * a.ldx + k, a.xtype) : 0.0f;
        }
        int count = 0;
#pragma unroll
        for (int i = 0; i < TESTS; ++i) {
            const unsigned long long nz = __ballot(x[i] != 0.0f);
            const int before = __popcll(nz & ((1ull << lane) - 1));
            if (x[i] != 0.0f) list[count + before] = Entry{x[i], k0 + i * 64 + lane};
            count += __popcll(nz);
        }
        if (count == 0) continue;
        // the last batch is filled up with its last row times 0
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        int group = -1;
        float sum[8] = {};
        uint2 scale = make_uint2(0u, 0u);
        const auto close = [&] {  // a group's sums, scaled
#pragma unroll
            for (int i = 0; i < 8; ++i)
                acc[i] = fmaf(sum[i] * factor, scale_value(((i < 4 ? scale.x : scale.y) >> (8 * (i & 3))) & 255u), acc[i]);
        };
        for (int base = 0; base < count; base += kFlight) {
            float xv[kFlight];
            int kv[kFlight];
            uint32_t q[kFlight];
            uint2 sc[kFlight];
            const Entry mine = list[base + lane < count ? base + lane : count - 1];
#pragma unroll
            for (int i = 0; i < kFlight; ++i) {
                kv[i] = __builtin_amdgcn_readlane(mine.k, i);
                xv[i] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine.x), i));
                const uint8_t *g = w + static_cast<int64_t>(kv[i] >> 5) * 17 * np;
                sc[i] = *reinterpret_cast<const uint2 *>(g + n0);
                q[i] = *reinterpret_cast<const uint32_t *>(g + np + (kv[i] & 31) * (np / 2) + n0 / 2);
            }
#pragma unroll
            for (int i = 0; i < kFlight; ++i) {
                if (base + i >= count) break;
                if (kv[i] >> 5 != group) {
                    if (group >= 0) close();
                    group = kv[i] >> 5;
                    scale = sc[i];
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum[c] = 0.0f;
                }
                add_row(sum, q[i], xv[i]);
            }
        }
        close();
        __builtin_amdgcn_wave_barrier();  // the list is read before the next turn writes it
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

// The ranges' sums: 64 outputs a workgroup, each of its wavefronts a quarter of
// the ranges in order, eight loads in flight; then the quarters in order.
__global__ void __launch_bounds__(256) w4_ranges_kernel(W4Args a, int ranges) {
    __shared__ float s[4][64];
    const int lane = threadIdx.x & 63, quarter = threadIdx.x >> 6;
    const int64_t all = static_cast<int64_t>(a.T) * a.w.N;
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 64 + lane;
    const float *p = a.part + (i < all ? i : all - 1);
    const int first = ranges * quarter / 4, last = ranges * (quarter + 1) / 4;
    float v = 0.0f;
    for (int r = first; r < last; r += 8) {
        float u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = p[static_cast<int64_t>(r + j < last ? r + j : r) * all];
#pragma unroll
        for (int j = 0; j < 8; ++j) v += r + j < last ? u[j] : 0.0f;
    }
    s[quarter][lane] = v;
    __syncthreads();
    if (quarter == 0 && i < all)
        store_as(a.y, i / a.w.N * a.ldy + i % a.w.N, s[0][lane] + s[1][lane] + s[2][lane] + s[3][lane], a.ytype);
}

}  // namespace

namespace {

// How the inputs of a call are cut: 64 `tests` inputs a turn of a wavefront, as
// many as leave it 4096 turns (8192 outputs of 32768 inputs, a twentieth nonzero,
// us at 1, 2 and 4 tests: one token 12.2 10.4 11.4, four 22.2 19.2 18.3; 4096 of
// 4096, a tenth: one token 6.9 7.9 10.8); a turn for every wavefront, up to 1024
// workgroups.
struct Cut {
    int tests, ranges;
};
Cut cut_of(const W4Shape &w, int T, int slots) {
    const int64_t cols = (w.np() + kOutputs - 1) / kOutputs * (T > 0 ? T : 1);
    const auto turns = [&](int tests) {
        return (w.K + tests * 64 - 1) / (tests * 64) * static_cast<int64_t>(slots ? slots : 1);
    };
    int tests = 4;
    while (tests > 1 && turns(tests) * cols < 4096) tests /= 2;
    const int64_t most = (turns(tests) + kWaves - 1) / kWaves;
    int64_t ranges = 1024 / cols;
    if (ranges > most) ranges = most;
    if (ranges > 64) ranges = 64;
    return {tests, ranges < 1 ? 1 : static_cast<int>(ranges)};
}

}  // namespace

int w4_skip_ranges(const W4Shape &w, int T, int slots) { return cut_of(w, T, slots).ranges; }

hipError_t launch_w4_skip(const W4Args &a, hipStream_t s) {
    const Cut cut = cut_of(a.w, a.T, a.slots);
    const dim3 grid(static_cast<unsigned>((a.w.np() + kOutputs - 1) / kOutputs * a.T), static_cast<unsigned>(cut.ranges));
    if (cut.tests == 1)
        w4_skip_kernel<1><<<grid, dim3(64 * kWaves), 0, s>>>(a, cut.ranges);
    else if (cut.tests == 2)
        w4_skip_kernel<2><<<grid, dim3(64 * kWaves), 0, s>>>(a, cut.ranges);
    else
        w4_skip_kernel<4><<<grid, dim3(64 * kWaves), 0, s>>>(a, cut.ranges);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || cut.ranges == 1) return e;
    const int64_t all = static_cast<int64_t>(a.T) * a.w.N;
    w4_ranges_kernel<<<dim3(static_cast<unsigned>((all + 63) / 64)), dim3(256), 0, s>>>(a, cut.ranges);
    return hipGetLastError();
}

}  // namespace isc
