// Products on 4-bit weights for a rectified x, its zeros skipped:
//   y[t][n] = sum over slots j of weight[t][j] * sum over k with x != 0 of w[n][k] x[t][j][k]
//
// The convolution's step on a matrix: a wavefront tests 64 inputs or more by
// ballots and lists the nonzeros in LDS, then reads one contiguous row of weights for
// each, five rows in flight, lanes running over outputs.  The bytes moved are the
// nonzeros' rows and the scales of the groups of 32 inputs that hold one.  A weight
// is widened under its own scale, so a row takes the same steps whether or not the
// one before was of its group: 28 vector instructions for its eight outputs a lane
// (57 where a group's sums were closed and scaled).  Sums are fp32, a slot's
// weighted once.
//
// The inputs (of all a token's slots) are cut into ranges, a workgroup each;
// its wavefronts take 64 TESTS inputs in turn.  Their sums meet in LDS in order, the
// ranges' in a second launch, so a result does not depend on timing.
//
// With few tokens a chain of waits bounds it (the inputs, the rows, the sums, the
// second launch): 8192 outputs of 32768 inputs, a twentieth nonzero, one token, take
// 12.0 us for 13.6 MB (9.7 us on the GPU alone), and 8 tokens of 8 experts, 2048
// outputs of 1408 with a tenth nonzero, 12.9 us for 13 MB.  With many the vector
// instructions do: 16 tokens of the first 40.3 us.  Five rows in flight leave room
// for eight wavefronts a unit; with eight rows it is 46.5 us, with three 40.0, and
// with half of the inputs nonzero 222, 219 and 236 us for five, eight and three.
#include "ffn.hpp"

namespace isc {
namespace {

constexpr int kWaves = 8;
constexpr int kOutputs = 512;  // outputs of a workgroup: eight a lane
constexpr int kFlight = 5;     // rows in flight

// Four outputs' products of one input: each weight widened under its own group's
// scale, whose byte stands in the exponent of a word (the conversion reads nothing
// else of it), then one multiply-add.  HALF: which four of the word of eight.
template <int HALF>
__device__ __forceinline__ void add_four(float *sum, uint32_t w, uint32_t scales, float x) {
    sum[0] = fmaf(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, __uint_as_float(scales << 23), 2 * HALF)[0], x, sum[0]);
    sum[1] = fmaf(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, __uint_as_float(scales << 15), 2 * HALF)[1], x, sum[1]);
    sum[2] = fmaf(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, __uint_as_float(scales << 7), 2 * HALF + 1)[0], x, sum[2]);
    sum[3] = fmaf(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, __uint_as_float(scales >> 1), 2 * HALF + 1)[1], x, sum[3]);
}

// A nonzero: its value and where its weights are, in half padded rows from the
// turn's first group on: the codes in the low half, the group's scales in the high.
struct Entry {
    float x;
    uint32_t at;
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
    const uint32_t n0 = static_cast<uint32_t>(c0 + lane * 8 < np ? c0 + lane * 8 : np - 8);
    const uint32_t half = static_cast<uint32_t>(np / 2);
    Entry *list = lists[wave];
    float acc[8] = {}, sum[8] = {};  // `sum`: of the slots under one weight
    float factor = 1.0f;
    int slot = -1;
    const auto close = [&] {  // a slot's sums, weighted
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            acc[i] = fmaf(sum[i], factor, acc[i]);
            sum[i] = 0.0f;
        }
    };
    for (int64_t turn = static_cast<int64_t>(range) * kWaves + wave; turn < turns;
         turn += static_cast<int64_t>(ranges) * kWaves) {
        const int j = static_cast<int>(turn / per), k0 = static_cast<int>(turn % per) * (TESTS * 64);
        const int64_t row = t * slots + j;
        // all tests' inputs on their way before anything waits
        uint32_t raw[TESTS];
        if (a.xtype == ISC_F32) {
            const uint32_t *p = static_cast<const uint32_t *>(a.x) + row * a.ldx;
#pragma unroll
            for (int i = 0; i < TESTS; ++i) raw[i] = p[k0 + i * 64 + lane < a.w.K ? k0 + i * 64 + lane : a.w.K - 1];
        } else {
            const uint16_t *p = static_cast<const uint16_t *>(a.x) + row * a.ldx;
#pragma unroll
            for (int i = 0; i < TESTS; ++i) raw[i] = p[k0 + i * 64 + lane < a.w.K ? k0 + i * 64 + lane : a.w.K - 1];
        }
        const uint8_t *w = a.packed;
        float weight = 1.0f;
        if (a.slots) {
            const int e = __builtin_amdgcn_readfirstlane(a.ids[row]);
            if (e < 0 || e >= a.w.E) continue;
            weight = a.weights[row];
            w += static_cast<int64_t>(e) * a.w.row_bytes();
        }
        float x[TESTS];
#pragma unroll
        for (int i = 0; i < TESTS; ++i) {
            x[i] = a.xtype == ISC_F16 ? F16::widen(raw[i]) : __uint_as_float(a.xtype == ISC_BF16 ? raw[i] << 16 : raw[i]);
            if (k0 + i * 64 + lane >= a.w.K) x[i] = 0.0f;
        }
        int count = 0;
#pragma unroll
        for (int i = 0; i < TESTS; ++i) {
            const unsigned long long nz = __ballot(x[i] != 0.0f);
            const int before = __popcll(nz & ((1ull << lane) - 1));
            const uint32_t group = static_cast<uint32_t>(i * 2 + (lane >> 5)) * 34u;  // 32 inputs and their scales
            if (x[i] != 0.0f) list[count + before] = Entry{x[i], group << 16 | (group + 2u + (lane & 31))};
            count += __popcll(nz);
        }
        if (count == 0) continue;
        if (j != slot) {
            if (slot >= 0) close();
            slot = j;
            factor = weight;
        }
        // the last batch is filled up with zeros, whose weights are set to 0 too
        if (lane < kFlight) list[count + lane] = Entry{0.0f, 0u};
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const uint8_t *from = w + static_cast<int64_t>(k0 >> 5) * 17 * np;
        for (int base = 0; base < count; base += kFlight) {
            float xv[kFlight];
            uint32_t q[kFlight];
            uint2 sc[kFlight];
#pragma unroll
            for (int i = 0; i < kFlight; ++i) {
                const Entry e = list[base + i];
                xv[i] = e.x;
                q[i] = *reinterpret_cast<const uint32_t *>(from + (__umul24(e.at & 0xffffu, half) + n0 / 2));
                sc[i] = *reinterpret_cast<const uint2 *>(from + (__umul24(e.at >> 16, half) + n0));
            }
            __builtin_amdgcn_sched_barrier(0);
            if (base + kFlight > count) {
#pragma unroll
                for (int i = 1; i < kFlight; ++i)
                    if (base + i >= count) q[i] = 0u, sc[i] = make_uint2(0u, 0u);
            }
#pragma unroll
            for (int i = 0; i < kFlight; ++i) {
                add_four<0>(sum, q[i], sc[i].x, xv[i]);
                add_four<1>(sum + 4, q[i], sc[i].y, xv[i]);
            }
        }
        __builtin_amdgcn_wave_barrier();  // the list is read before the next turn writes it
    }
    close();
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
    const int64_t cols = (a.w.np() + kOutputs - 1) / kOutputs;
    const int64_t most = kLaunchThreads / (64 * kWaves) / cols;  // tokens of a launch
    const int64_t xb = a.xtype == ISC_F32 ? 4 : 2, yb = a.ytype == ISC_F32 ? 4 : 2, slots = a.slots ? a.slots : 1;
    for (int64_t t0 = 0; t0 < a.T; t0 += most) {  // (once where there are ranges, of a thousand workgroups at most)
        W4Args part = a;
        part.T = static_cast<int>(a.T - t0 < most ? a.T - t0 : most);
        part.x = past(a.x, t0 * slots * a.ldx * xb), part.y = past(a.y, t0 * a.ldy * yb);
        part.ids = past(a.ids, t0 * slots * 4), part.weights = past(a.weights, t0 * slots * 4);
        const dim3 grid(static_cast<unsigned>(cols * part.T), static_cast<unsigned>(cut.ranges));
        if (cut.tests == 1)
            w4_skip_kernel<1><<<grid, dim3(64 * kWaves), 0, s>>>(part, cut.ranges);
        else if (cut.tests == 2)
            w4_skip_kernel<2><<<grid, dim3(64 * kWaves), 0, s>>>(part, cut.ranges);
        else
            w4_skip_kernel<4><<<grid, dim3(64 * kWaves), 0, s>>>(part, cut.ranges);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (cut.ranges == 1) return hipSuccess;
    const int64_t all = static_cast<int64_t>(a.T) * a.w.N;
    w4_ranges_kernel<<<dim3(static_cast<unsigned>((all + 63) / 64)), dim3(256), 0, s>>>(a, cut.ranges);
    return hipGetLastError();
}

}  // namespace isc
