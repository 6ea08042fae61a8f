// Root-mean-square norm with the residual's addition, and its gradient.
//
//   h = x + r,  rstd = (mean(h^2) + eps)^(-1/2),  y = h rstd w
//
// One workgroup per row, the row in registers (up to 32768 values), so x and r
// are read once: eight consecutive values per thread and chunk, a group of 32
// outputs (the 8-bit form's unit) in four neighbouring lanes.  Sums are fp32; h
// is normalised as it was added, before its rounding to x's type.  Memory bounds
// it: 8192 rows of 8192 in bfloat16 with residual and 8-bit output move 472 MB in
// 86 us, 5.5 TB/s; one row of 4096 takes 3.2 us on the GPU, all of it waits.  Rows
// of one wavefront have a workgroup each too: four or eight of them in one were no
// faster (16384 rows of 512 12.2 us against 12.9 and 13.2).
//
// The gradient, with n = h rstd and g = dy w:
//   dx = rstd (g - n mean(g n)) + dh,   dw = sum over rows of dy n
// A workgroup walks rows and keeps its columns' sums of dy n in registers;
// the workgroups' sums are added in order by a second launch.  8192 rows of 4096
// in bfloat16 move 268 MB in 59 us, 4.6 TB/s; 777 rows of 1155 in fp32 take 9.7 us,
// two launches and a few rows one after another.
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
    // by halves: the wavefronts' values are of one size, and so are their pairs'
    float t[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] = i < waves ? sums[i] : 0.0f;
#pragma unroll
    for (int n = 8; n > 0; n >>= 1)
#pragma unroll
        for (int i = 0; i < n; ++i) t[i] += t[i + n];
    return t[0];
}

// m^(-1/2) to half a unit in the last place and a little: the instruction's
// value, and a Newton step on its error.  The 8-bit form's values move by whole
// steps where the last bit does.
__device__ __forceinline__ float reciprocal_root(float m) {
    const float r = __builtin_amdgcn_rsqf(m);
    const float h = m * r, low = fmaf(m, r, -h);
    const float e = fmaf(-low, r, fmaf(-h, r, 1.0f));
    const float better = fmaf(0.5f * r, e, r);
    return fabsf(better) < __builtin_inff() ? better : r;  // 0 and infinity have no error to take off
}

constexpr int kShortRows = 8;  // rows of one wavefront that a workgroup of the gradient takes at once

// First of the eight values of a row that a thread holds in chunk c.  SHORT: a
// wavefront holds the row.
template <bool SHORT = false>
__device__ __forceinline__ int at(int c) {
    return SHORT ? static_cast<int>(threadIdx.x & 63) * 8
                 : (c * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * 8;
}

// Chunk c of a row of D values, 0 where there are none.  RAGGED, for 16-bit types
// and a D over 8 that is no multiple of it: the row's last values come with one wide
// load of the eight before its end and are moved to their places without a branch,
// so that their wavefront has all tensors' loads in flight together like the others
// (3000 bfloat16 rows of 3351: norm 16.8 us, value by value 24.9; gradient 24.1 and
// 44.0).  Not where a thread holds several chunks (3000 rows of 8195: 56.7 and 55.2,
// gradient 70.1 and 71.1), nor for fp32, whose values do not wait to be widened one
// by one (3548 rows of 3351: 38.3 and 37.1, gradient 47.9 and 39.6).
template <class T, bool SHORT = false, bool RAGGED = false>
__device__ __forceinline__ void load_chunk(float (&v)[8], const typename T::type *row, int c, int D) {
    if constexpr (!RAGGED || sizeof(typename T::type) == 4) {  // (a weight may be fp32)
        load8<T>(v, row + at<SHORT>(c), D - at<SHORT>(c));
    } else {
        const int here = at<SHORT>(c), from = here < D - 8 ? here : D - 8, by = here - from;
        const uint4 a = load_any<uint4>(row + from);
        uint32_t w0 = a.x, w1 = a.y, w2 = a.z, w3 = a.w;
        if (by & 4) w0 = w2, w1 = w3, w2 = 0u, w3 = 0u;
        if (by & 2) w0 = w1, w1 = w2, w2 = w3, w3 = 0u;
        const uint32_t half = by & 1 ? 16 : 0, all = by < 8 ? 0xffffffffu : 0u;
        const uint32_t w[4] = {__builtin_amdgcn_alignbit(w1, w0, half) & all, __builtin_amdgcn_alignbit(w2, w1, half) & all,
                               __builtin_amdgcn_alignbit(w3, w2, half) & all, __builtin_amdgcn_alignbit(0u, w3, half) & all};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = T::widen(w[i] & 0xffffu);
            v[2 * i + 1] = T::widen(w[i] >> 16);
        }
    }
}
template <class T, bool SHORT = false>
__device__ __forceinline__ void store_chunk(typename T::type *row, const float (&v)[8], int c, int D) {
    store8<T>(row + at<SHORT>(c), v, D - at<SHORT>(c));
}
template <bool SHORT = false, bool RAGGED = false>
__device__ __forceinline__ void load_weight(float (&w)[8], const void *p, int c, int D, int type) {
    if (type == ISC_F32)
        load_chunk<F32, SHORT, RAGGED>(w, static_cast<const float *>(p), c, D);
    else if (type == ISC_BF16)
        load_chunk<BF16, SHORT, RAGGED>(w, static_cast<const uint16_t *>(p), c, D);
    else
        load_chunk<F16, SHORT, RAGGED>(w, static_cast<const uint16_t *>(p), c, D);
}

// The 8-bit form of a chunk of outputs.  A group's largest magnitude is taken
// as bits, under which NaN comes out above everything.
__device__ __forceinline__ void store_mx8(uint8_t *q, uint8_t *scales, const float (&v)[8], int c, int D) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = op_max(m, __float_as_uint(v[j]) & 0x7fffffffu);
    m = op_max(m, dpp<0xb1, 0xf>(m, m));              // quad_perm 1,0,3,2
    m = op_max(m, dpp<0x4e, 0xf>(m, m));              // quad_perm 2,3,0,1
    const uint32_t b = group_scale<8, 0x600000u>(m);  // 448 = 1.75 * 2^8
    const float inv = __uint_as_float((254u - (b > 253u ? 253u : b)) << 23);
    uint32_t lo = 0x7f7f7f7fu, hi = 0x7f7f7f7fu;
    if (b != 255u) {
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, 0, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, hi, true);
    }
    const int n = D - at(c);
    if (n >= 8) {
        store_any(q + at(c), make_uint2(lo, hi));
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) q[at(c) + j] = static_cast<uint8_t>((j < 4 ? lo : hi) >> (8 * (j & 3)));
    }
    if ((threadIdx.x & 3) == 0 && at(c) < D) scales[at(c) / 32] = static_cast<uint8_t>(b);
}

template <class T, int C, bool RAGGED>
__global__ void __launch_bounds__(1024) rmsnorm_kernel(NormArgs a) {
    using E = typename T::type;
    __shared__ float sums[16];
    const int64_t t = blockIdx.x;
    float v[C][8], w[C][8];
    float ss = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) load_chunk<T, false, RAGGED>(v[c], static_cast<const E *>(a.x) + t * a.ldx, c, a.D);
    if (a.r) {
        float u[C][8];
#pragma unroll
        for (int c = 0; c < C; ++c) load_chunk<T, false, RAGGED>(u[c], static_cast<const E *>(a.r) + t * a.ldr, c, a.D);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] += u[c][j];
    }
    // short rows: the weight on its way while the sum is taken
    if (C <= 2)
#pragma unroll
        for (int c = 0; c < C; ++c) load_weight<false, RAGGED>(w[c], a.w, c, a.D, a.wtype);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(v[c][j], v[c][j], ss);
    if (a.h)
#pragma unroll
        for (int c = 0; c < C; ++c) store_chunk<T>(static_cast<E *>(a.h) + t * a.ldh, v[c], c, a.D);
    const float mean = block_sum(ss, sums) / static_cast<float>(a.D);
    const float rstd = reciprocal_root(mean + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[t] = rstd;
    if (!a.y && !a.q) return;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (C > 2) load_weight<false, RAGGED>(w[c], a.w, c, a.D, a.wtype);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c][j] = at(c) + j < a.D ? v[c][j] * rstd * w[c][j] : 0.0f;
        if (a.y) store_chunk<T>(static_cast<E *>(a.y) + t * a.ldy, v[c], c, a.D);
        if (a.q)
            store_mx8(static_cast<uint8_t *>(a.q) + t * a.ldq, static_cast<uint8_t *>(a.scales) + t * a.lds, v[c],
                             c, a.D);
    }
}

// Rows that the registers do not hold: read once for the sum and, from the
// cache, once more for the outputs.  Nothing is written before the second
// reading, so h may still stand in for x or r.
template <class T>
__global__ void __launch_bounds__(1024) rmsnorm_long_kernel(NormArgs a, int chunks) {
    using E = typename T::type;
    __shared__ float sums[16];
    const int64_t t = blockIdx.x;
    const auto load = [&](float(&v)[8], int c) {
        load_chunk<T>(v, static_cast<const E *>(a.x) + t * a.ldx, c, a.D);
        if (!a.r) return;
        float u[8];
        load_chunk<T>(u, static_cast<const E *>(a.r) + t * a.ldr, c, a.D);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += u[j];
    };
    float ss = 0.0f;
    for (int c = 0; c < chunks; ++c) {
        float v[8];
        load(v, c);
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(v[j], v[j], ss);
    }
    const float mean = block_sum(ss, sums) / static_cast<float>(a.D);
    const float rstd = reciprocal_root(mean + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[t] = rstd;
    for (int c = 0; c < chunks; ++c) {
        float v[8], w[8];
        load(v, c);
        load_weight(w, a.w, c, a.D, a.wtype);
        if (a.h) store_chunk<T>(static_cast<E *>(a.h) + t * a.ldh, v, c, a.D);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = at(c) + j < a.D ? v[j] * rstd * w[j] : 0.0f;
        if (a.y) store_chunk<T>(static_cast<E *>(a.y) + t * a.ldy, v, c, a.D);
        if (a.q)
            store_mx8(static_cast<uint8_t *>(a.q) + t * a.ldq, static_cast<uint8_t *>(a.scales) + t * a.lds, v, c, a.D);
    }
}

// SHORT: rows of one wavefront, as many at once as the workgroup has wavefronts;
// else one row at a time.  A row is on its way while the one before is worked on,
// where the registers hold both (C of 1).
template <class T, int C, bool SHORT, bool RAGGED>
__global__ void __launch_bounds__(1024) rmsnorm_bwd_kernel(NormBwdArgs a) {
    using E = typename T::type;
    __shared__ float sums[2][16];
    __shared__ float joined[SHORT ? kShortRows : 1][SHORT ? 512 : 1];
    const int wave = threadIdx.x >> 6;
    const int64_t step = SHORT ? static_cast<int64_t>(gridDim.x) * kShortRows : gridDim.x;
    float w[C][8], acc[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        load_weight<SHORT, RAGGED>(w[c], a.w, c, a.D, a.wtype);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[c][j] = 0.0f;
    }
    // a row of h, dy and dh, as loaded
    const auto load = [&](int64_t t, float(&n)[C][8], float(&g)[C][8], float(&d)[C][8], float &rstd) {
        if (t >= a.T) return;
        rstd = a.rstd[t];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            load_chunk<T, SHORT, RAGGED>(n[c], static_cast<const E *>(a.h) + t * a.ldh, c, a.D);
            load_chunk<T, SHORT, RAGGED>(g[c], static_cast<const E *>(a.dy) + t * a.ldy, c, a.D);
            if (a.dh)
                load_chunk<T, SHORT, RAGGED>(d[c], static_cast<const E *>(a.dh) + t * a.ldd, c, a.D);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) d[c][j] = 0.0f;
        }
    };
    const int64_t t0 = SHORT ? static_cast<int64_t>(blockIdx.x) * kShortRows + wave : blockIdx.x;
    float nn[C][8], ng[C][8], nd[C][8], nr = 0.0f;  // the next row
    if constexpr (C == 1) load(t0, nn, ng, nd, nr);
    int turn = 0;
    for (int64_t t = t0; t < a.T; t += step, turn ^= 1) {
        float n[C][8], g[C][8], d[C][8], rstd = nr;
        if constexpr (C == 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) n[0][j] = nn[0][j], g[0][j] = ng[0][j], d[0][j] = nd[0][j];
        } else {
            load(t, n, g, d, rstd);
        }
        float dot = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                n[c][j] *= rstd;
                acc[c][j] = fmaf(g[c][j], n[c][j], acc[c][j]);
                g[c][j] *= w[c][j];
                dot = fmaf(g[c][j], n[c][j], dot);
            }
        // (dx may be one of the tensors that are read: row t is in registers now, and
        // row t + step is no other row's output)
        if constexpr (C == 1) load(t + step, nn, ng, nd, nr);
        // two sets of sums in turn: a row's are read before the row after the
        // next overwrites them, with the barrier of the row between
        const float mean = (SHORT ? wave_sum(dot) : block_sum(dot, sums[turn])) / static_cast<float>(a.D);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = fmaf(rstd, fmaf(-n[c][j], mean, g[c][j]), d[c][j]);
            store_chunk<T, SHORT>(static_cast<E *>(a.dx) + t * a.ldx, o, c, a.D);
        }
    }
    float *part = a.part + static_cast<int64_t>(blockIdx.x) * a.D;
    if constexpr (SHORT) {
#pragma unroll
        for (int j = 0; j < 8; ++j) joined[wave][at<SHORT>(0) + j] = acc[0][j];
        __syncthreads();
        for (int i = threadIdx.x; i < a.D; i += blockDim.x) {
            float u = 0.0f;
#pragma unroll
            for (int r = 0; r < kShortRows; ++r) u += joined[r][i];
            part[i] = u;
        }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c) store_chunk<F32>(part, acc[c], c, a.D);
    }
}

// dw[i] = sum of part[b][i] over b: 32 columns a workgroup, each of its 32 half
// wavefronts every 32nd row, eight loads in flight; then the halves in order.
__global__ void __launch_bounds__(1024) column_sum_kernel(const float *part, int rows, int D, float *dw) {
    __shared__ float s[32][33];
    const int lane = threadIdx.x & 31, half = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + lane;
    const float *p = part + (i < D ? i : D - 1);
    float t = 0.0f;
    for (int b = half; b < rows; b += 256) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = p[static_cast<int64_t>(b + 32 * j < rows ? b + 32 * j : b) * D];
#pragma unroll
        for (int j = 0; j < 8; ++j) t += b + 32 * j < rows ? v[j] : 0.0f;
    }
    s[half][lane] = t;
    __syncthreads();
    if (half == 0 && i < D) {
        float u = 0.0f;
#pragma unroll
        for (int h = 0; h < 32; ++h) u += s[h][lane];
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

// Whether a row's last values are moved to their places (load_chunk).
template <class T>
bool ragged(int D) {
    return sizeof(typename T::type) == 2 && D % 8 != 0 && D > 8;
}

template <class T>
hipError_t norm_of(const NormArgs &a, hipStream_t s) {
    const RowPlan p = row_plan(a.D, 1024);
    const dim3 grid(static_cast<unsigned>(a.T)), block(static_cast<unsigned>(p.threads));
    switch (p.chunks) {
    case 1:
        if (ragged<T>(a.D))
            rmsnorm_kernel<T, 1, true><<<grid, block, 0, s>>>(a);
        else
            rmsnorm_kernel<T, 1, false><<<grid, block, 0, s>>>(a);
        break;
    case 2: rmsnorm_kernel<T, 2, false><<<grid, block, 0, s>>>(a); break;
    case 4: rmsnorm_kernel<T, 4, false><<<grid, block, 0, s>>>(a); break;
    default: rmsnorm_long_kernel<T><<<grid, block, 0, s>>>(a, p.chunks); break;
    }
    return hipGetLastError();
}

template <class T>
hipError_t norm_bwd_of(const NormBwdArgs &a, hipStream_t s) {
    const RowPlan p = row_plan(a.D, 1024);
    const bool brief = p.threads == 64;
    const int blocks = norm_bwd_blocks(a.T, a.D);
    const dim3 grid(static_cast<unsigned>(blocks)), block(static_cast<unsigned>(brief ? 64 * kShortRows : p.threads));
    const bool uneven = ragged<T>(a.D);
    if (brief && uneven)
        rmsnorm_bwd_kernel<T, 1, true, true><<<grid, block, 0, s>>>(a);
    else if (brief)
        rmsnorm_bwd_kernel<T, 1, true, false><<<grid, block, 0, s>>>(a);
    else if (p.chunks == 1 && uneven)
        rmsnorm_bwd_kernel<T, 1, false, true><<<grid, block, 0, s>>>(a);
    else if (p.chunks == 1)
        rmsnorm_bwd_kernel<T, 1, false, false><<<grid, block, 0, s>>>(a);
    else
        rmsnorm_bwd_kernel<T, 2, false, false><<<grid, block, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    column_sum_kernel<<<dim3(static_cast<unsigned>((a.D + 31) / 32)), dim3(1024), 0, s>>>(a.part, blocks, a.D, a.dw);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs &a, hipStream_t s) {
    return a.type == ISC_F32 ? norm_of<F32>(a, s) : a.type == ISC_BF16 ? norm_of<BF16>(a, s) : norm_of<F16>(a, s);
}

int norm_bwd_blocks(int T, int D) {
    const int threads = row_plan(D, 1024).threads;
    const int turns = threads == 64 ? (T + kShortRows - 1) / kShortRows : T;
    // Short rows want more workgroups at once, long ones fewer sums for the second
    // launch to read (8192 bfloat16 rows, us with 1, 2, 4, 8 workgroups a compute
    // unit: of 1024 52.6 31.0 22.4 21.9, of 2048 78.7 46.7 33.2 37.8, of 4096 89.1
    // 59.8 62.6 71.0, of 8192 116 118 126 142); two turns each at least, the second's
    // loads ahead, from 256 turns on (rows of 4096: 330 of them 9.7 and 10.6 with one
    // each, 200 of them 8.2 and 8.1), from 512 of short rows' (2400 rows of 500: 11.2
    // and 10.2).
    const int most = 256 * (threads > 512 ? 1 : threads > 256 || threads == 64 ? 2 : threads > 128 ? 4 : 8);
    const int some = turns < (threads == 64 ? 512 : 256) ? turns : (turns + 1) / 2;
    return some < 1 ? 1 : some < most ? some : most;
}

hipError_t launch_rmsnorm_bwd(const NormBwdArgs &a, hipStream_t s) {
    return a.type == ISC_F32    ? norm_bwd_of<F32>(a, s)
           : a.type == ISC_BF16 ? norm_bwd_of<BF16>(a, s)
                                : norm_bwd_of<F16>(a, s);
}

}  // namespace isc
