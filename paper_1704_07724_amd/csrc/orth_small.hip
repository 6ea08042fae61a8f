// Orthogonalising matrices of which one side is at most 64 (orthogonalize.hip says what is
// computed, and what is held how): a launch a step.
//
// A = X X^T (or X^T X) is one 64 x 64 tile, so a step needs no more of other workgroups
// than their parts of it.  A workgroup adds up all parts of A, makes b A + c A^2,
// multiplies its blocks of 64 along the longer side by it, four at a time by four
// wavefronts each, and leaves its part of the next A.  Every workgroup reads every part, 16
// KiB each, so parts are few: with one for each block, adding them up took half of a step.
// They have two places, in turn, since others still read the last ones.
// A matrix of few rows has few singular values, over which the errors of fp16 operands
// do not average (2 x 3: 1.4e-2 of the result after five steps, 64 x 300 2.7e-3), so here every
// operand is held as the state is, in two parts, of whose products three are kept (2.6e-5,
// 1.4e-5).  They cost a ninth of the time (2048 x 64 57 us in one part), for twice as many LDS
// reads, which are what a block takes.
// What bounds it: a launch's start and end and one chain of loads a step: 2048 x
// 64 takes 64 us in seven launches (85 as products of their own, in 23).
#include "orthogonalize.hpp"

#include "tile_product.hpp"

namespace isc {
namespace {

using namespace tp;

// Values as the state holds them: each an fp16 value and, times 2^11, what that leaves.
template <int N>
struct Split {
    uint32_t high[N / 2], low[N / 2];
    __device__ __forceinline__ void of(const float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            uint32_t h[2], l[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                h[k] = F16::narrow(v[2 * i + k]);
                l[k] = F16::narrow((v[2 * i + k] - F16::widen(h[k])) * kOrthLow);
            }
            high[i] = h[0] | h[1] << 16;
            low[i] = l[0] | l[1] << 16;
        }
    }
    __device__ __forceinline__ void join(float (&v)[N]) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = fmaf(F16::widen(i & 1 ? low[i / 2] >> 16 : low[i / 2] & 0xffffu), 1.0f / kOrthLow,
                        F16::widen(i & 1 ? high[i / 2] >> 16 : high[i / 2] & 0xffffu));
    }
};

// 64 x 64 values in LDS, the second parts behind the first ones; chunks of 16 bytes placed so
// that reads along the rows and transposing ones meet all banks.
struct Square {
    static constexpr int kPart = 64 * 128, kBytes = 2 * kPart;
    static __device__ __forceinline__ int at(int row, int c) { return (row * 8 + (c ^ (row >> 1 & 7))) * 16; }
    // 8 consecutive values of a row
    static __device__ __forceinline__ void store(char *lds, int row, int c, const Split<8> &v) {
        char *to = lds + at(row, c);
        *reinterpret_cast<uint4 *>(to) = make_uint4(v.high[0], v.high[1], v.high[2], v.high[3]);
        *reinterpret_cast<uint4 *>(to + kPart) = make_uint4(v.low[0], v.low[1], v.low[2], v.low[3]);
    }
    static __device__ __forceinline__ Split<8> load(const char *lds, int row, int c) {
        const uint4 h = *reinterpret_cast<const uint4 *>(lds + at(row, c));
        const uint4 l = *reinterpret_cast<const uint4 *>(lds + at(row, c) + kPart);
        return Split<8>{{h.x, h.y, h.z, h.w}, {l.x, l.y, l.z, l.w}};
    }
    // A matrix operand as Stage::operand() gives it, of indices o to o + 32: rows, or columns (SIDE
    // kAcross), over inner indices 16 * kk to 16 * kk + 16.
    template <Side SIDE, bool DEALT>
    static __device__ __forceinline__ s16x8 operand(const char *lds, int o, int kk, int lane) {
        const int h = lane >> 5;
        if constexpr (SIDE == kAlong) {
            const int m = lane & 31, row = o + (DEALT ? 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3) : m);
            return *reinterpret_cast<const s16x8 *>(lds + at(row, 2 * kk + h));
        } else {
            const int i = lane & 15, u = 4 * ((lane >> 4) & 1) + (i & 3);
            const int c = o + 4 * (DEALT ? 4 * (u & 1) + (u >> 1) : u);
            s16x4 v[2];
#pragma unroll
            for (int q = 0; q < 2; ++q)
                v[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(
                    lds + at(16 * kk + 8 * h + 4 * q + (i >> 2), c >> 3) + (c & 7) * 2));
            return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// Adds the 32 x 32 tile at (i, j) of a product of two squares over 64 inner indices: lane l has
// row i + l % 32, columns j + 16 * (l / 32) on.  The products with a second part add up by
// themselves; two second parts' is 2^-22 of a term and left out.
template <Side XS, Side WS>
__device__ __forceinline__ void multiply(f32x16 &acc, const char *x, const char *w, int i, int j, int lane) {
    f32x16 low = {};
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
        const s16x8 w0 = Square::operand<WS, true>(w, j, kk, lane), x0 = Square::operand<XS, false>(x, i, kk, lane);
        acc = mfma<F16>(w0, x0, acc);
        low = mfma<F16>(w0, Square::operand<XS, false>(x + Square::kPart, i, kk, lane), low);
        low = mfma<F16>(Square::operand<WS, true>(w + Square::kPart, j, kk, lane), x0, low);
    }
#pragma unroll
    for (int n = 0; n < 16; ++n) acc[n] = fmaf(low[n], 1.0f / kOrthLow, acc[n]);
}

struct SmallStep {
    OrthArgs a;
    int step;      // -1: only the first A
    float c[3];
    const float *from;  // parts of A, each 64 x 64
    float *to;
};

// G's type T matters to the launches that read it.
template <class T, bool WIDE>
__global__ __launch_bounds__(1024) void orth_small_kernel(const SmallStep p) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const OrthShape &s = p.a.s;
    const int parts = s.parts(), n = blockIdx.x / parts, part = blockIdx.x % parts, np = s.np();
    const int tid = threadIdx.x, lane = tid & 63, wave = (tid >> 6) & 3, group = tid >> 8;
    const int wi = wave >> 1 << 5, wj = (wave & 1) << 5;
    // this thread's 16 values of every square, in LDS, in memory and of the products
    const int row = wi + (lane & 31), col = wj + 16 * (lane >> 5);
    const int blocks = static_cast<int>((s.span() + 63) / 64);
    const bool first = p.step <= 0, last = p.step + 1 == p.a.steps;
    double by = 0.0;  // as a double: the inverse of a small norm may be beyond fp32
    if (first)
        by = orth_inverse_norm(reinterpret_cast<const double *>(p.a.ws), n, s.blocks(), p.a.eps,
                               reinterpret_cast<double *>(lds + Square::kBytes));
    uint16_t *high = reinterpret_cast<uint16_t *>(p.a.ws + s.operand(0)) + n * s.of_state(),
             *low = reinterpret_cast<uint16_t *>(p.a.ws + s.low()) + n * s.of_state();
    char *square = lds, *poly = lds + Square::kBytes, *x = lds + (2 + group) * Square::kBytes;
    if (p.step >= 0) {
        const float *from = p.from + static_cast<int64_t>(n) * parts * 4096 + tid * 4;
        float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll 8
        for (int q = 0; q < parts; ++q) {
            const float4 u = *reinterpret_cast<const float4 *>(from + q * 4096);
            sum.x += u.x;
            sum.y += u.y;
            sum.z += u.z;
            sum.w += u.w;
        }
        Split<4> all;
        all.of({sum.x, sum.y, sum.z, sum.w});
        char *to = square + Square::at(tid >> 4, (tid & 15) >> 1) + (tid & 1) * 8;
        *reinterpret_cast<uint2 *>(to) = make_uint2(all.high[0], all.high[1]);
        *reinterpret_cast<uint2 *>(to + Square::kPart) = make_uint2(all.low[0], all.low[1]);
        __syncthreads();
        if (group == 0) {
            f32x16 acc = {};
            multiply<kAlong, kAlong>(acc, square, square, wi, wj, lane);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float v[8];
                Split<8> u = Square::load(square, row, col / 8 + q);
                u.join(v);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = fmaf(p.c[1], v[k], p.c[2] * (acc[8 * q + k] * (1.0f / kOrthUp)));
                u.of(v);
                Square::store(poly, row, col / 8 + q, u);
            }
        }
    }
    f32x16 sums = {};
    // past the last block there is nothing to multiply, but all wavefronts meet as often
    for (int b0 = 4 * part; b0 < blocks; b0 += 4 * parts) {
        const int b = b0 + group;
        // the block's rows and columns in memory
        const int r = WIDE ? row : 64 * b + row, c = WIDE ? 64 * b + col : col;
        Split<8> held[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int there = r < s.M ? s.N - c - 8 * q : 0;
            if (first) {
                float u[8], v[8];
                Raw8<T> g;
                g.load(static_cast<const typename T::type *>(p.a.g) + (static_cast<int64_t>(n) * s.M + r) * p.a.ldg + c + 8 * q,
                       there);
                g.widen(u);
#pragma unroll
                for (int k = 0; k < 8; ++k)  // inf * 0 is no zero
                    v[k] = k < there ? static_cast<float>(static_cast<double>(u[k]) * by) * kOrthUp : 0.0f;
                held[q].of(v);
            } else {
                Raw8<F16> hi, lo;
                hi.load(high + static_cast<int64_t>(r) * np + c + 8 * q, there > 0 ? 8 : 0);
                lo.load(low + static_cast<int64_t>(r) * np + c + 8 * q, there > 0 ? 8 : 0);
                held[q] = {{hi.a.x, hi.a.y, hi.a.z, hi.a.w}, {lo.a.x, lo.a.y, lo.a.z, lo.a.w}};
            }
        }
        __syncthreads();  // the last block's reads are done, and the polynomial is there
#pragma unroll
        for (int q = 0; q < 2; ++q) Square::store(x, row, col / 8 + q, held[q]);
        if (p.step >= 0) {
            __syncthreads();
            f32x16 acc = {};
            if (b < blocks) {
            if (WIDE)
                multiply<kAlong, kAcross>(acc, poly, x, wi, wj, lane);
            else
                multiply<kAlong, kAlong>(acc, x, poly, wi, wj, lane);
            }
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int there = r < s.M ? s.N - c - 8 * q : 0;
                float v[8];
                held[q].join(v);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[k] = fmaf(p.c[0], v[k], acc[8 * q + k] * (1.0f / kOrthUp)) * (last ? 1.0f / kOrthUp : 1.0f);
                    v[k] = k < there ? v[k] : 0.0f;
                }
                if (last) {
                    if (there > 0)
                        store8_as(p.a.o, (static_cast<int64_t>(n) * s.M + r) * p.a.ldo + c + 8 * q, v, there, p.a.otype);
                    continue;
                }
                held[q].of(v);
                if (there <= 0) continue;
                const int64_t place = static_cast<int64_t>(r) * np + c + 8 * q;
                store_any(high + place, make_uint4(held[q].high[0], held[q].high[1], held[q].high[2], held[q].high[3]));
                store_any(low + place, make_uint4(held[q].low[0], held[q].low[1], held[q].low[2], held[q].low[3]));
            }
            if (last) continue;
            __syncthreads();  // the products have read the old values
#pragma unroll
            for (int q = 0; q < 2; ++q) Square::store(x, row, col / 8 + q, held[q]);
        }
        __syncthreads();
        if (b < blocks) {
        if (WIDE)
            multiply<kAlong, kAlong>(sums, x, x, wi, wj, lane);
        else
            multiply<kAcross, kAcross>(sums, x, x, wi, wj, lane);
        }
    }
    if (last) return;
    // the four blocks' sums, in order; 2^6 times A, as its fp16 operand is
    __syncthreads();
    float4 *others = reinterpret_cast<float4 *>(lds);
    if (group)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            others[(4 * (group - 1) + i) * 256 + (tid & 255)] = make_float4(sums[4 * i], sums[4 * i + 1], sums[4 * i + 2], sums[4 * i + 3]);
    __syncthreads();
    if (group) return;
    float *to = p.to + (static_cast<int64_t>(n) * parts + part) * 4096 + row * 64 + col;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float4 sum = make_float4(sums[4 * i], sums[4 * i + 1], sums[4 * i + 2], sums[4 * i + 3]);
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            const float4 u = others[(4 * q + i) * 256 + tid];
            sum.x += u.x;
            sum.y += u.y;
            sum.z += u.z;
            sum.w += u.w;
        }
        *reinterpret_cast<float4 *>(to + 4 * i) =
            make_float4(sum.x * (1.0f / kOrthUp), sum.y * (1.0f / kOrthUp), sum.z * (1.0f / kOrthUp), sum.w * (1.0f / kOrthUp));
    }
}

template <class T>
hipError_t launch_steps(const OrthArgs &a, hipStream_t s) {
    float *parts = reinterpret_cast<float *>(a.ws + a.s.partial());
    const int64_t all = static_cast<int64_t>(a.s.B) * a.s.parts();
    const auto kernel = a.s.wide() ? orth_small_kernel<T, true> : orth_small_kernel<T, false>;
    constexpr int kLds = 6 * Square::kBytes;
    if (hipError_t e = a.s.wide() ? allow_lds<orth_small_kernel<T, true>>(kLds) : allow_lds<orth_small_kernel<T, false>>(kLds);
        e != hipSuccess)
        return e;
    for (int step = -1; step < a.steps; ++step) {
        SmallStep p{a, step, {0.0f, 0.0f, 0.0f}, parts + (step & 1) * all * 4096, parts + ((step + 1) & 1) * all * 4096};
        for (int i = 0; step >= 0 && i < 3; ++i) p.c[i] = a.coef[3 * step + i];
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(all)), dim3(1024), kLds, s, p);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_orth_small(const OrthArgs &a, hipStream_t s) {
    return a.type == ISC_F32 ? launch_steps<F32>(a, s) : a.type == ISC_BF16 ? launch_steps<BF16>(a, s) : launch_steps<F16>(a, s);
}

}  // namespace isc
