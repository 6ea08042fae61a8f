// Root-mean-square norm with the residual's addition, and its gradient.
//
//   h = x + r,  rstd = (mean(h^2) + eps)^(-1/2),  y = h rstd w
//
// One workgroup per row, the row in registers (up to 32768 values), so x and r
// are read once: eight consecutive values per thread and chunk, a group of 32
// outputs (the 8-bit form's unit) in four neighbouring lanes.  Sums are fp32; h
// is normalised as it was added, before its rounding to x's type.  Memory bounds
// it: 8192 rows of 8192 in bfloat16 with residual and 8-bit output move 472 MB in
// 85 us, 5.5 TB/s; one row of 4096 takes 3.0 us on the GPU, all of it waits.  Rows
// of one wavefront have a workgroup each too: four or eight of them in one were no
// faster (16384 rows of 512 12.2 us against 12.9 and 13.2).
//
// The gradient, with n = h rstd and g = dy w:
//   dx = rstd (g - n mean(g n)) + dh,   dw = sum over rows of dy n
// A workgroup walks rows and keeps its columns' sums of dy n in registers;
// the workgroups' sums are added in order by a second launch.  8192 rows of 4096
// in bfloat16 move 268 MB in 50 us, 5.4 TB/s; 777 rows of 1155 in fp32 take 9.5 us,
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
// steps where the last bit does.  The instruction takes what is below 2^-126 for 0, so
// that is raised by 2^48 first.
__device__ __forceinline__ float reciprocal_root(float m) {
    const bool small = m < 0x1p-126f;
    m *= small ? 0x1p48f : 1.0f;
    const float r = __builtin_amdgcn_rsqf(m);
    const float h = m * r, low = fmaf(m, r, -h);
    const float e = fmaf(-low, r, fmaf(-h, r, 1.0f));
    const float better = fmaf(0.5f * r, e, r);
    // 0 and infinity have no error to take off
    return (fabsf(better) < __builtin_inff() ? better : r) * (small ? 0x1p24f : 1.0f);
}

constexpr int kShortRows = 8;  // rows of one wavefront that a workgroup of the gradient takes at once

// First of the eight values of a row that a thread holds in chunk c.  SHORT: a
// wavefront holds the row.
template <bool SHORT = false>
__device__ __forceinline__ int at(int c) {
    return SHORT ? static_cast<int>(threadIdx.x & 63) * 8
                 : (c * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x)) * 8;
}

// How a thread's eight values of a row are read.  kEven, for widths that are a
// multiple of 8, and kMoved, for other widths over 8 of 16-bit types: one wide load
// without a branch, from the eight values before the row's end where the thread's own
// would pass it, and what is the thread's taken out of it when the values are used.
// So the loads of all tensors, and of the row after, are in flight together: behind a
// branch each waits to be widened before the next is sent.  kAny: value by value at
// the row's end.
// (8192 bfloat16 rows of 4096, gradient: 50.4 us, each load behind its branch 59.4;
// 3000 rows of 3351: norm 16.4, value by value 24.9, gradient 22.7 and 44.0.)  Not
// for rows of several chunks that end inside eight (3000 rows of 8195: norm 56.7 and
// 55.2), nor the gradient of fp32, whose values need no widening to wait for.
enum Reading { kAny, kEven, kMoved };

using Words = uint32_t[8];  // eight values as loaded; 16-bit ones take half of them

template <class T, Reading READ, bool SHORT = false>
struct Chunk {
    static constexpr bool kWide = sizeof(typename T::type) == 4;
    static constexpr Reading kRead = kWide && READ == kMoved ? kAny : READ;  // (a weight beside 16-bit values)

    // Chunk c of a row of D values.
    static __device__ __forceinline__ void load(Words &w, const typename T::type *row, int c, int D) {
        if constexpr (kRead == kAny) {
            float v[8];
            load8<T>(v, row + at<SHORT>(c), D - at<SHORT>(c));
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[i]);
        } else {
            const int here = at<SHORT>(c);
            const typename T::type *p = row + (here < D - 8 ? here : D - 8);
            const uint4 a = load_any<uint4>(p);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
            if constexpr (kWide) {
                const uint4 b = load_any<uint4>(p + 4);
                w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
            }
        }
    }

    // Its values, 0 past the row's end.
    static __device__ __forceinline__ void get(float (&v)[8], const Words &w, int c, int D) {
        if constexpr (kRead == kAny) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        } else if constexpr (kWide) {
            const bool there = at<SHORT>(c) < D;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = there ? __uint_as_float(w[i]) : 0.0f;
        } else {
            const int here = at<SHORT>(c), by = here < D - 8 ? 0 : here - (D - 8);
            uint32_t u[4] = {w[0], w[1], w[2], w[3]};
            if constexpr (kRead == kMoved) {
                move_down(u, by);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = by < 8 ? u[i] : 0u;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = T::widen(u[i] & 0xffffu);
                v[2 * i + 1] = T::widen(u[i] >> 16);
            }
        }
    }
};

// The same of the weight, whose type is known at run time.
template <Reading READ, bool SHORT = false>
struct WeightChunk {
    static __device__ __forceinline__ void load(Words &w, const void *p, int c, int D, int type) {
        if (type == ISC_F32)
            Chunk<F32, READ, SHORT>::load(w, static_cast<const float *>(p), c, D);
        else if (READ != kAny || type == ISC_BF16)  // (fp16 as well, unless it is widened at once)
            Chunk<BF16, READ, SHORT>::load(w, static_cast<const uint16_t *>(p), c, D);
        else
            Chunk<F16, READ, SHORT>::load(w, static_cast<const uint16_t *>(p), c, D);
    }
    static __device__ __forceinline__ void get(float (&v)[8], const Words &w, int c, int D, int type) {
        if (type == ISC_F32)
            Chunk<F32, READ, SHORT>::get(v, w, c, D);
        else if (type == ISC_BF16)
            Chunk<BF16, READ, SHORT>::get(v, w, c, D);
        else
            Chunk<F16, READ, SHORT>::get(v, w, c, D);
    }
};

template <class T>
__device__ __forceinline__ void load_chunk(float (&v)[8], const typename T::type *row, int c, int D) {
    load8<T>(v, row + at(c), D - at(c));
}
template <class T, bool SHORT = false>
__device__ __forceinline__ void store_chunk(typename T::type *row, const float (&v)[8], int c, int D) {
    store8<T>(row + at<SHORT>(c), v, D - at<SHORT>(c));
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

template <class T, int C, Reading READ>
__global__ void __launch_bounds__(1024) rmsnorm_kernel(NormArgs a) {
    using E = typename T::type;
    __shared__ float sums[16];
    const int64_t t = blockIdx.x;
    float v[C][8], w[C][8];
    float ss = 0.0f;
    using In = Chunk<T, READ>;
    using Weight = WeightChunk<READ>;
    Words x[C], r[C], weight[C];
#pragma unroll
    for (int c = 0; c < C; ++c) In::load(x[c], static_cast<const E *>(a.x) + t * a.ldx, c, a.D);
    if (a.r)
#pragma unroll
        for (int c = 0; c < C; ++c) In::load(r[c], static_cast<const E *>(a.r) + t * a.ldr, c, a.D);
    // short rows: the weight on its way while the sum is taken
    if (C <= 2)
#pragma unroll
        for (int c = 0; c < C; ++c) Weight::load(weight[c], a.w, c, a.D, a.wtype);
#pragma unroll
    for (int c = 0; c < C; ++c) In::get(v[c], x[c], c, a.D);
    if (a.r)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float u[8];
            In::get(u, r[c], c, a.D);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] += u[j];
        }
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
        if (C > 2) Weight::load(weight[c], a.w, c, a.D, a.wtype);
        Weight::get(w[c], weight[c], c, a.D, a.wtype);
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
        Words weight;
        WeightChunk<kAny>::load(weight, a.w, c, a.D, a.wtype);
        WeightChunk<kAny>::get(w, weight, c, a.D, a.wtype);
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
template <class T, int C, bool SHORT, Reading READ>
__global__ void __launch_bounds__(1024) rmsnorm_bwd_kernel(NormBwdArgs a) {
    using E = typename T::type;
    __shared__ float sums[2][16];
    __shared__ float joined[SHORT ? kShortRows : 1][SHORT ? 512 : 1];
    const int wave = threadIdx.x >> 6;
    const int64_t step = SHORT ? static_cast<int64_t>(gridDim.x) * kShortRows : gridDim.x;
    float w[C][8], acc[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        Words weight;
        WeightChunk<READ, SHORT>::load(weight, a.w, c, a.D, a.wtype);
        WeightChunk<READ, SHORT>::get(w[c], weight, c, a.D, a.wtype);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[c][j] = 0.0f;
    }
    // chunk c of a row of h, dy and dh as loaded, and dh's values
    using In = Chunk<T, READ, SHORT>;
    const auto load = [&](int64_t t, int c, Words &h, Words &dy, Words &dh) {
        In::load(h, static_cast<const E *>(a.h) + t * a.ldh, c, a.D);
        In::load(dy, static_cast<const E *>(a.dy) + t * a.ldy, c, a.D);
        if (a.dh)
            In::load(dh, static_cast<const E *>(a.dh) + t * a.ldd, c, a.D);
        else if (READ == kAny)
#pragma unroll
            for (int i = 0; i < 8; ++i) dh[i] = 0u;
    };
    const auto get_dh = [&](int c, const Words &dh, float(&d)[8]) {
        if (READ == kAny || a.dh)  // (the one set 0 where there is none, the other not even loaded)
            In::get(d, dh, c, a.D);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = 0.0f;
    };
    const int64_t t0 = SHORT ? static_cast<int64_t>(blockIdx.x) * kShortRows + wave : blockIdx.x;
    constexpr bool kAhead = C == 1;  // the next row is on its way
    Words next_h, next_dy, next_dh;
    float next_rstd = 0.0f;
    if (kAhead && t0 < a.T) {
        next_rstd = a.rstd[t0];
        load(t0, 0, next_h, next_dy, next_dh);
    }
    int turn = 0;
    for (int64_t t = t0; t < a.T; t += step, turn ^= 1) {
        float n[C][8], g[C][8], d[C][8];
        // dh of two chunks stays as loaded until it is added, half the registers of its
        // values, which would spill (8192 bfloat16 rows of 8200 119 us, 125 with spills,
        // 2000 fp16 rows of 12288 38 and 42); one chunk has room for them
        Words dh[C];
        const float rstd = kAhead ? next_rstd : a.rstd[t];
        if constexpr (kAhead) {
            In::get(n[0], next_h, 0, a.D);
            In::get(g[0], next_dy, 0, a.D);
            get_dh(0, next_dh, d[0]);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                Words h, dy;
                load(t, c, h, dy, dh[c]);
                In::get(n[c], h, c, a.D);
                In::get(g[c], dy, c, a.D);
            }
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
        if (kAhead && t + step < a.T) {
            next_rstd = a.rstd[t + step];
            load(t + step, 0, next_h, next_dy, next_dh);
        }
        // two sets of sums in turn: a row's are read before the row after the
        // next overwrites them, with the barrier of the row between
        const float mean = (SHORT ? wave_sum(dot) : block_sum(dot, sums[turn])) / static_cast<float>(a.D);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float o[8];
            if (!kAhead) get_dh(c, dh[c], d[c]);
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

template <class T>
constexpr bool kHalf = sizeof(typename T::type) == 2;

template <class T, int C>
void norm_with(const NormArgs &a, dim3 grid, dim3 block, hipStream_t s) {
    if (a.D % 8 == 0) {
        rmsnorm_kernel<T, C, kEven><<<grid, block, 0, s>>>(a);
        return;
    }
    if constexpr (kHalf<T> && C == 1)
        if (a.D > 8) {
            rmsnorm_kernel<T, C, kMoved><<<grid, block, 0, s>>>(a);
            return;
        }
    rmsnorm_kernel<T, C, kAny><<<grid, block, 0, s>>>(a);
}

// (fp32 by kAny alone: 3000 rows of 2048 take 22.2 us, by kEven 23.9)
template <class T, int C, bool SHORT>
void norm_bwd_with(const NormBwdArgs &a, dim3 grid, dim3 block, hipStream_t s) {
    if constexpr (kHalf<T>) {
        if (a.D % 8 == 0) {
            rmsnorm_bwd_kernel<T, C, SHORT, kEven><<<grid, block, 0, s>>>(a);
            return;
        }
        if constexpr (C == 1)
            if (a.D > 8) {
                rmsnorm_bwd_kernel<T, C, SHORT, kMoved><<<grid, block, 0, s>>>(a);
                return;
            }
    }
    rmsnorm_bwd_kernel<T, C, SHORT, kAny><<<grid, block, 0, s>>>(a);
}

// Rows t0 .. t0 + n of a call.
NormArgs rows_of(NormArgs a, int64_t t0, int64_t n, int64_t size) {
    a.x = past(a.x, t0 * a.ldx * size), a.r = past(a.r, t0 * a.ldr * size);
    a.h = past(a.h, t0 * a.ldh * size), a.y = past(a.y, t0 * a.ldy * size);
    a.q = past(a.q, t0 * a.ldq), a.scales = past(a.scales, t0 * a.lds);
    a.rstd = past(a.rstd, t0 * 4);
    a.T = static_cast<int>(n);
    return a;
}

template <class T>
hipError_t norm_of(const NormArgs &all, hipStream_t s) {
    const RowPlan p = row_plan(all.D, 1024);
    // 2^26 - 1 rows of up to 512 values a launch, 2^22 - 1 from 7681 on
    const int64_t most = kLaunchThreads / p.threads;
    for (int64_t t0 = 0; t0 < all.T; t0 += most) {
        const int64_t n = all.T - t0 < most ? all.T - t0 : most;
        const NormArgs a = rows_of(all, t0, n, sizeof(typename T::type));
        const dim3 grid(static_cast<unsigned>(n)), block(static_cast<unsigned>(p.threads));
        switch (p.chunks) {
        case 1: norm_with<T, 1>(a, grid, block, s); break;
        case 2: norm_with<T, 2>(a, grid, block, s); break;
        case 4: norm_with<T, 4>(a, grid, block, s); break;
        default: rmsnorm_long_kernel<T><<<grid, block, 0, s>>>(a, p.chunks); break;
        }
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T>
hipError_t norm_bwd_of(const NormBwdArgs &a, hipStream_t s) {
    const RowPlan p = row_plan(a.D, 1024);
    const bool brief = p.threads == 64;
    // without rows there are no sums to add: dw is 0, and the weight, which such a call
    // need not have, is not read
    const int blocks = a.T > 0 ? norm_bwd_blocks(a.T, a.D) : 0;
    if (blocks > 0) {
        const dim3 grid(static_cast<unsigned>(blocks)), block(static_cast<unsigned>(brief ? 64 * kShortRows : p.threads));
        if (brief)
            norm_bwd_with<T, 1, true>(a, grid, block, s);
        else if (p.chunks == 1)
            norm_bwd_with<T, 1, false>(a, grid, block, s);
        else
            norm_bwd_with<T, 2, false>(a, grid, block, s);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    column_sum_kernel<<<dim3(static_cast<unsigned>((a.D + 31) / 32)), dim3(1024), 0, s>>>(a.part, blocks, a.D, a.dw);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs &a, hipStream_t s) {
    return a.type == ISC_F32 ? norm_of<F32>(a, s) : a.type == ISC_BF16 ? norm_of<BF16>(a, s) : norm_of<F16>(a, s);
}

int norm_bwd_blocks(int T, int D) {
    const int threads = row_plan(D, 1024).threads;
    const int64_t turns = threads == 64 ? (int64_t{T} + kShortRows - 1) / kShortRows : T;  // (T may be 2^31 - 1)
    // Short rows want more workgroups at once, long ones fewer sums for the second
    // launch to read (8192 bfloat16 rows, us with 1, 2, 4, 8 workgroups a compute
    // unit: of 1024 37.6 24.0 20.0 21.6, of 2048 50.1 33.9 31.8 35.6, of 4096 58.7
    // 50.8 55.3 62.3, of 8192 103 107 116 132, and of 512, eight at once, 10.7 11.4
    // 11.4 11.4; 1024 rows of 4096 13.6 15.4 15.5 15.5); two turns each at least, the
    // second's loads ahead, from 256 turns on (rows of 4096: 330 of them 9.7 and 10.6
    // with one each, 200 of them 8.2 and 8.1), from 512 of short rows' (2400 rows of
    // 500: 11.2 and 10.2).
    const int64_t most = 256 * (threads == 64 || threads > 512 || (threads > 256 && turns < 2048) ? 1 : threads > 256 ? 2 : 4);
    const int64_t some = turns < (threads == 64 ? 512 : 256) ? turns : (turns + 1) / 2;
    return static_cast<int>(some < 1 ? 1 : some < most ? some : most);
}

hipError_t launch_rmsnorm_bwd(const NormBwdArgs &a, hipStream_t s) {
    return a.type == ISC_F32    ? norm_bwd_of<F32>(a, s)
           : a.type == ISC_BF16 ? norm_bwd_of<BF16>(a, s)
                                : norm_bwd_of<F16>(a, s);
}

}  // namespace isc
