// Root-mean-square norm with the residual's addition, and its gradient.
//
//   h = x + r,  rstd = (mean(h^2) + eps)^(-1/2),  y = h rstd w
//
// One workgroup per row, the row in registers: eight consecutive values per
// thread and chunk, so x and r are read once, and a group of 32 outputs (the
// 8-bit form's unit) lies in four neighbouring lanes.  Sums are fp32; h is
// normalised as it was added, before its rounding to x's type.
//
// The gradient, with n = h rstd and g = dy w:
//   dx = rstd (g - n mean(g n)) + dh,   dw = sum over rows of dy n
// A workgroup walks rows and keeps its columns' sums of dy n in registers;
// the workgroups' sums are added in order by a second launch.
#include "ffn.hpp"

namespace isc {
namespace {

// Sum over the workgroup, in every thread; `sums` holds one value per wavefront.
__device__ __forceinline__ float block_sum(float v, float *sums) {
    v = wave_sum(v);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
    __syncthreads();
    float t = 0.0f;
    for (int i = 0; i < waves; ++i) t += sums[i];
    return t;
}

__device__ __forceinline__ void load_weight8(float (&w)[8], const void *p, int64_t i, int n, int type, bool whole) {
    if (type == ISC_F32)
        load8<F32>(w, static_cast<const float *>(p) + i, n, whole);
    else if (type == ISC_BF16)
        load8<BF16>(w, static_cast<const uint16_t *>(p) + i, n, whole);
    else
        load8<F16>(w, static_cast<const uint16_t *>(p) + i, n, whole);
}

template <class T, int C>
__global__ void __launch_bounds__(1024) rmsnorm_kernel(NormArgs a) {
    using E = typename T::type;
    __shared__ float sums[16];
    const int64_t t = blockIdx.x;
    const E *x = static_cast<const E *>(a.x) + t * a.ldx;
    const E *r = a.r ? static_cast<const E *>(a.r) + t * a.ldr : nullptr;
    float v[C][8];
    float ss = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int i = (c * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * 8;
        const int n = a.D - i;
        if (n > 0) {
            load8<T>(v[c], x + i, n, a.whole);
            if (r) {
                float u[8];
                load8<T>(u, r + i, n, a.whole);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] += u[j];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = 0.0f;
        }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(v[c][j], v[c][j], ss);
    if (a.h) {
        E *h = static_cast<E *>(a.h) + t * a.ldh;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int i = (c * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * 8;
            if (i < a.D) store8<T>(h + i, v[c], a.D - i, a.whole);
        }
    }
    const float mean = block_sum(ss, sums) / static_cast<float>(a.D);
    const float rstd = 1.0f / sqrtf(mean + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[t] = rstd;
    if (!a.y && !a.q) return;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int i = (c * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * 8;
        const int n = a.D - i;
        float w[8];
        if (n > 0)
            load_weight8(w, a.w, i, n, a.wtype, a.whole);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] = n > j ? v[c][j] * rstd * w[j] : 0.0f;
        if (a.y && n > 0) store8<T>(static_cast<E *>(a.y) + t * a.ldy + i, v[c], n, a.whole);
        if (!a.q) continue;
        // four lanes hold a group; its largest magnitude as bits, under which
        // NaN comes out above everything
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = op_max(m, __float_as_uint(v[c][j]) & 0x7fffffffu);
        m = op_max(m, dpp<0xb1, 0xf>(m, m));  // quad_perm 1,0,3,2
        m = op_max(m, dpp<0x4e, 0xf>(m, m));  // quad_perm 2,3,0,1
        const uint32_t b = group_scale<8, 0x600000u>(m);  // 448 = 1.75 * 2^8
        const float inv = __uint_as_float((254u - (b > 253u ? 253u : b)) << 23);
        uint32_t lo = 0x7f7f7f7fu, hi = 0x7f7f7f7fu;
        if (b != 255u) {
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[c][0] * inv, v[c][1] * inv, 0, false);
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[c][2] * inv, v[c][3] * inv, lo, true);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[c][4] * inv, v[c][5] * inv, 0, false);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[c][6] * inv, v[c][7] * inv, hi, true);
        }
        if (n <= 0) continue;
        uint8_t *q = static_cast<uint8_t *>(a.q) + t * a.ldq + i;
        if (a.whole) {
            *reinterpret_cast<uint2 *>(q) = make_uint2(lo, hi);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) q[j] = static_cast<uint8_t>((j < 4 ? lo : hi) >> (8 * (j & 3)));
        }
        if ((threadIdx.x & 3) == 0) static_cast<uint8_t *>(a.scales)[t * a.lds + i / 32] = static_cast<uint8_t>(b);
    }
}

template <class T, int C>
__global__ void __launch_bounds__(1024) rmsnorm_bwd_kernel(NormBwdArgs a) {
    using E = typename T::type;
    __shared__ float sums[2][16];
    float w[C][8], acc[C][8];
    const auto at = [](int c) { return (c * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * 8; };
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[c][j] = acc[c][j] = 0.0f;
        if (at(c) < a.D) load_weight8(w[c], a.w, at(c), a.D - at(c), a.wtype, a.whole);
    }
    int turn = 0;
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x, turn ^= 1) {
        const E *h = static_cast<const E *>(a.h) + t * a.ldh;
        const E *dy = static_cast<const E *>(a.dy) + t * a.ldy;
        const E *dh = a.dh ? static_cast<const E *>(a.dh) + t * a.ldd : nullptr;
        const float rstd = a.rstd[t];
        float n[C][8], g[C][8], d[C][8];
        float dot = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll
            for (int j = 0; j < 8; ++j) n[c][j] = g[c][j] = d[c][j] = 0.0f;
            if (at(c) < a.D) {
                load8<T>(n[c], h + at(c), a.D - at(c), a.whole);
                load8<T>(g[c], dy + at(c), a.D - at(c), a.whole);
                if (dh) load8<T>(d[c], dh + at(c), a.D - at(c), a.whole);
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                n[c][j] *= rstd;
                acc[c][j] = fmaf(g[c][j], n[c][j], acc[c][j]);
                g[c][j] *= w[c][j];
                dot = fmaf(g[c][j], n[c][j], dot);
            }
        // two sets of sums in turn: a row's are read before the row after the
        // next overwrites them, with the barrier of the row between
        const float mean = block_sum(dot, sums[turn]) / static_cast<float>(a.D);
        E *dx = static_cast<E *>(a.dx) + t * a.ldx;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (at(c) >= a.D) continue;
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = fmaf(rstd, fmaf(-n[c][j], mean, g[c][j]), d[c][j]);
            store8<T>(dx + at(c), o, a.D - at(c), a.whole);
        }
    }
    float *part = a.part + static_cast<int64_t>(blockIdx.x) * a.D;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (at(c) + j < a.D) part[at(c) + j] = acc[c][j];
}

// dw[i] = sum of part[b][i] over b: 64 columns a workgroup, 16 wavefronts
// each a sixteenth of the rows, in order.
__global__ void __launch_bounds__(1024) column_sum_kernel(const float *part, int rows, int D, float *dw) {
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int i = blockIdx.x * 64 + lane;
    float t = 0.0f;
    if (i < D)
        for (int b = wave; b < rows; b += 16) t += part[static_cast<int64_t>(b) * D + i];
    s[wave][lane] = t;
    __syncthreads();
    if (wave == 0 && i < D) {
        float u = 0.0f;
#pragma unroll
        for (int w = 0; w < 16; ++w) u += s[w][lane];
        dw[i] = u;
    }
}

// Threads of a row's workgroup, and chunks of eight values each holds.
struct RowPlan {
    int threads, chunks;
};
RowPlan row_plan(int D, int most) {
    const int eights = (D + 7) / 8;
    int threads = (eights + 63) / 64 * 64;
    if (threads > most) threads = most;
    int chunks = 1;
    while (chunks * threads < eights) chunks *= 2;
    return {threads, chunks};
}

template <class T>
hipError_t norm_of(const NormArgs &a, hipStream_t s) {
    const RowPlan p = row_plan(a.D, 1024);
    const dim3 grid(static_cast<unsigned>(a.T)), block(static_cast<unsigned>(p.threads));
    switch (p.chunks) {
    case 1: rmsnorm_kernel<T, 1><<<grid, block, 0, s>>>(a); break;
    case 2: rmsnorm_kernel<T, 2><<<grid, block, 0, s>>>(a); break;
    case 4: rmsnorm_kernel<T, 4><<<grid, block, 0, s>>>(a); break;
    default: rmsnorm_kernel<T, 8><<<grid, block, 0, s>>>(a); break;
    }
    return hipGetLastError();
}

template <class T>
hipError_t norm_bwd_of(const NormBwdArgs &a, hipStream_t s) {
    const RowPlan p = row_plan(a.D, 1024);
    const int blocks = norm_bwd_blocks(a.T, a.D);
    const dim3 grid(static_cast<unsigned>(blocks)), block(static_cast<unsigned>(p.threads));
    switch (p.chunks) {
    case 1: rmsnorm_bwd_kernel<T, 1><<<grid, block, 0, s>>>(a); break;
    default: rmsnorm_bwd_kernel<T, 2><<<grid, block, 0, s>>>(a); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    column_sum_kernel<<<dim3(static_cast<unsigned>((a.D + 63) / 64)), dim3(1024), 0, s>>>(a.part, blocks, a.D, a.dw);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs &a, hipStream_t s) {
    return a.type == ISC_F32 ? norm_of<F32>(a, s) : a.type == ISC_BF16 ? norm_of<BF16>(a, s) : norm_of<F16>(a, s);
}

int norm_bwd_blocks(int T, int D) {
    const int threads = row_plan(D, 1024).threads;
    const int most = 256 * (2048 / threads < 4 ? 2048 / threads : 4);
    return T < most ? (T < 1 ? 1 : T) : most;
}

hipError_t launch_rmsnorm_bwd(const NormBwdArgs &a, hipStream_t s) {
    return a.type == ISC_F32    ? norm_bwd_of<F32>(a, s)
           : a.type == ISC_BF16 ? norm_bwd_of<BF16>(a, s)
                                : norm_bwd_of<F16>(a, s);
}

}  // namespace isc
