// Orthogonalising updates (isc_orthogonalize): X = G / (|G| + eps), |G| the
// Frobenius norm, then some steps of
//   X <- a X + (b A + c A^2) X,  A = X X^T     (A = X^T X from the right, where G is tall)
// an odd polynomial of X's singular values that leaves its singular vectors as
// they are and brings the values towards one.
//
// What is held how.  The state X is fp32: what a step adds to a small singular
// direction is small beside the large ones, and every later step magnifies an
// error there as it does the direction (3.4^5 = 480 in all), so a state in 16 bits
// loses 2^-6 of a gradient with few strong directions.  The operands of the
// products, X, A and b A + c A^2, are fp16, whose errors stay where the operand is
// one factor among fp32 sums: 1e-3 at most of the result's norm, as much as its
// own rounding to bf16 (fp64 against it: 704 x 2048, noise over 16 directions,
// 1.1e-4; noise alone 1.5e-3).  Operands are scaled by 2^6 on their way to fp16,
// which keeps entries of 2^-14 normal and any that the coefficients' check lets
// through finite.
//
// A and b A + c A^2 are symmetric: tiles on and below the diagonal are computed,
// the others are their mirror images.  All matrices of a stack share each launch:
// three products a step.  What bounds it: the matrix cores.
#include "orthogonalize.hpp"

#include "tile_product.hpp"

namespace isc {
namespace {

using namespace tp;

constexpr float kUp = 64.0f;  // of every fp16 operand

struct OrthProduct {
    OrthShape s;
    Rows x, w;                      // the first matrix's
    int64_t xhop, whop;             // bytes to the next one's
    int inner, rows, cols;
    const uint16_t *square;         // A, where b A is added
    uint16_t *out16;                // fp16 results
    float *state;
    void *o;                        // the last step's results
    int64_t ldo;
    int otype;
    float a, b, c;
};

// Sums of squares, in fp64: no gradient's square leaves its range.
template <class T>
__global__ __launch_bounds__(256) void orth_norm_kernel(const OrthArgs a) {
    const OrthShape &s = a.s;
    const int64_t row0 = static_cast<int64_t>(blockIdx.y) * s.M;
    double sum = 0.0;
    const int groups = s.np() / 8;
    const int64_t all = static_cast<int64_t>(s.M) * groups, hop = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all; i += hop) {
        const int64_t r = i / groups;
        const int c = static_cast<int>(i - r * groups) * 8;
        float v[8];
        load8<T>(v, static_cast<const typename T::type *>(a.g) + (row0 + r) * a.ldg + c, s.N - c);
#pragma unroll
        for (int q = 0; q < 8; ++q) sum = fma(static_cast<double>(v[q]), static_cast<double>(v[q]), sum);
    }
    __shared__ double sums[256];
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int d = 128; d > 0; d /= 2) {
        if (threadIdx.x < static_cast<unsigned>(d)) sums[threadIdx.x] += sums[threadIdx.x + d];
        __syncthreads();
    }
    if (threadIdx.x == 0) reinterpret_cast<double *>(a.ws)[blockIdx.y * gridDim.x + blockIdx.x] = sums[0];
}

template <class T>
__global__ __launch_bounds__(256) void orth_scale_kernel(const OrthArgs a) {
    const OrthShape &s = a.s;
    const int64_t row0 = static_cast<int64_t>(blockIdx.y) * s.M;
    double sum = 0.0;
    for (int i = 0; i < s.blocks(); ++i) sum += reinterpret_cast<const double *>(a.ws)[blockIdx.y * s.blocks() + i];
    const double by = 1.0 / (sqrt(sum) + static_cast<double>(a.eps));
    float *state = reinterpret_cast<float *>(a.ws + s.state()) + blockIdx.y * s.of_state();
    uint16_t *operand = reinterpret_cast<uint16_t *>(a.ws + s.operand(0)) + blockIdx.y * s.of_state();
    const int groups = s.np() / 8;
    const int64_t all = static_cast<int64_t>(s.M) * groups, hop = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all; i += hop) {
        const int64_t r = i / groups;
        const int c = static_cast<int>(i - r * groups) * 8;
        float v[8];
        load8<T>(v, static_cast<const typename T::type *>(a.g) + (row0 + r) * a.ldg + c, s.N - c);
#pragma unroll
        for (int q = 0; q < 8; ++q)  // 0 * inf is no zero behind the last column
            v[q] = c + q < s.N ? static_cast<float>(static_cast<double>(v[q]) * by) : 0.0f;
        store8<F32>(state + r * s.np() + c, v, 8);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] *= kUp;
        store8<F16>(operand + r * s.np() + c, v, 8);
    }
}

enum Product { kGram, kPoly, kApply };

template <class TL, Product WHAT>
__global__ __launch_bounds__(TL::kThreads) void orth_product_kernel(const OrthProduct p) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int id = of_xcd(blockIdx.x, gridDim.x);
    const int down = (p.rows + TL::BI - 1) / TL::BI;
    int n, ti, tj;
    if constexpr (WHAT == kApply) {
        const int across = (p.cols + TL::BJ - 1) / TL::BJ;
        n = id / (down * across);
        ti = id / across % down;
        tj = id % across;
    } else {
        const int half = down * (down + 1) / 2;
        n = id / half;
        const int at = id % half;  // ti (ti + 1) / 2 + tj
        ti = static_cast<int>((__builtin_sqrtf(8.0f * at + 1.0f) - 1.0f) * 0.5f);
        if (ti * (ti + 1) / 2 > at) --ti;
        if ((ti + 1) * (ti + 2) / 2 <= at) ++ti;
        tj = at - ti * (ti + 1) / 2;
    }
    const int i0 = ti * TL::BI, j0 = tj * TL::BJ;
    Rows x = p.x, w = p.w;
    x.base += n * p.xhop;
    w.base += n * p.whop;
    TL t;
    t.run(x, w, i0, j0, p.inner, p.rows - i0, p.cols - j0, lds);
    if constexpr (WHAT == kApply) {
        const int np = p.s.np();
        float *state = p.state + n * p.s.of_state();
        t.each([&](int, int i, int j, const f32x16 &sums) {
            const int row = i0 + i, col = j0 + j;
            if (row >= p.rows || col >= p.cols) return;
            float *x = state + static_cast<int64_t>(row) * np + col;
            f32x16 v;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float u[8];
                load8<F32>(u, x + 8 * q, np - col - 8 * q);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    v[8 * q + k] = fmaf(p.a, u[k], sums[8 * q + k] * (1.0f / (kUp * kUp)));
            }
            if (p.o) {
                const int64_t at = (static_cast<int64_t>(n) * p.rows + row) * p.ldo + col;
                if (p.otype == ISC_BF16)
                    store16<BF16>(static_cast<uint16_t *>(p.o) + at, v, p.cols - col);
                else
                    store16<F16>(static_cast<uint16_t *>(p.o) + at, v, p.cols - col);
                return;
            }
            // behind the last column the operands' zeros made zeros, or another column's sums
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = col + k < p.cols ? v[k] : 0.0f;
            store16<F32>(x, v, np - col);
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] *= kUp;
            store16<F16>(p.out16 + n * p.s.of_state() + static_cast<int64_t>(row) * np + col, v, np - col);
        });
    } else {
        const int m = p.rows, mp = p.s.mp();
        uint16_t *out = p.out16 + n * p.s.of_square();
        const uint16_t *square = p.square + n * p.s.of_square();
        t.each([&](int, int i, int j, const f32x16 &sums) {
            const int row = i0 + i, col = j0 + j;
            if (row >= mp || col >= mp) return;
            f32x16 v;
            if constexpr (WHAT == kGram) {
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = sums[k] * (1.0f / kUp);
            } else {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float u[8] = {};
                    if (row < m) load8<F16>(u, square + static_cast<int64_t>(row) * mp + col + 8 * q, mp - col - 8 * q);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        v[8 * q + k] = fmaf(p.b, u[k], p.c * (sums[8 * q + k] * (1.0f / kUp)));
                }
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = row < m && col + k < m ? v[k] : 0.0f;
            if (row < m) store16<F16>(out + static_cast<int64_t>(row) * mp + col, v, mp - col);
            if (ti != tj) {
#pragma unroll
                for (int k = 0; k < 16; ++k)
                    if (col + k < m) store<F16>(out + static_cast<int64_t>(col + k) * mp + row, v[k]);
            }
        });
    }
}

template <class TL, Product WHAT>
hipError_t launch_product(const OrthProduct &p, hipStream_t s) {
    if (hipError_t e = allow_lds(orth_product_kernel<TL, WHAT>, TL::kLds); e != hipSuccess) return e;
    const int64_t down = (p.rows + TL::BI - 1) / TL::BI, across = (p.cols + TL::BJ - 1) / TL::BJ;
    const int64_t grid = p.s.B * (WHAT == kApply ? down * across : down * (down + 1) / 2);
    hipLaunchKernelGGL((orth_product_kernel<TL, WHAT>), dim3(static_cast<unsigned>(grid)), dim3(TL::kThreads), TL::kLds,
                       s, p);
    return hipGetLastError();
}

template <Side XS, Side WS, Product WHAT>
hipError_t launch_tile(const OrthProduct &p, hipStream_t s) {
    if constexpr (WHAT == kApply) return launch_product<Tile<F16, true, XS, WS, 256, 256, 2, 4>, WHAT>(p, s); else return launch_product<Tile<F16, true, XS, WS, 256, 256, 2, 4>, WHAT>(p, s);
}

template <class T>
hipError_t launch_state(const OrthArgs &a, hipStream_t s) {
    const dim3 grid(static_cast<unsigned>(a.s.blocks()), static_cast<unsigned>(a.s.B));
    hipLaunchKernelGGL(orth_norm_kernel<T>, grid, dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(orth_scale_kernel<T>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

bool orth_launches_fit(const OrthShape &s) {
    const int64_t down = (s.M + 127) / 128, across = (s.N + 127) / 128, m = (s.m() + 127) / 128;
    const int64_t most = down * across > m * (m + 1) / 2 ? down * across : m * (m + 1) / 2;
    return s.B * most * 256 <= kLaunchThreads;
}

hipError_t launch_orthogonalize(const OrthArgs &a, hipStream_t s) {
    const OrthShape &h = a.s;
    hipError_t e = a.type == ISC_F32    ? launch_state<F32>(a, s)
                   : a.type == ISC_BF16 ? launch_state<BF16>(a, s)
                                        : launch_state<F16>(a, s);
    if (e != hipSuccess) return e;
    uint16_t *square = reinterpret_cast<uint16_t *>(a.ws + h.square(0)),
             *poly = reinterpret_cast<uint16_t *>(a.ws + h.square(1));
    const int m = h.m(), np = h.np(), mp = h.mp();
    for (int i = 0; i < a.steps; ++i) {
        const char *x = a.ws + h.operand(i & 1);
        OrthProduct p{};
        p.s = h;
        p.a = a.coef[3 * i];
        p.b = a.coef[3 * i + 1];
        p.c = a.coef[3 * i + 2];
        p.rows = p.cols = m;
        p.xhop = p.whop = 2 * h.of_state();
        p.x = p.w = {x, int64_t{2} * np, nullptr, h.M, np};
        p.out16 = square;
        p.square = square;
        p.inner = h.wide() ? np : h.M;
        e = h.wide() ? launch_tile<kAlong, kAlong, kGram>(p, s) : launch_tile<kAcross, kAcross, kGram>(p, s);
        if (e != hipSuccess) return e;
        const Rows sq{reinterpret_cast<const char *>(square), int64_t{2} * mp, nullptr, m, mp};
        p.x = p.w = sq;
        p.xhop = p.whop = 2 * h.of_square();
        p.inner = mp;
        p.out16 = poly;
        if ((e = launch_tile<kAlong, kAlong, kPoly>(p, s)) != hipSuccess) return e;
        const Rows pl{reinterpret_cast<const char *>(poly), int64_t{2} * mp, nullptr, m, mp};
        const Rows st{x, int64_t{2} * np, nullptr, h.M, np};
        p.rows = h.M;
        p.cols = h.N;
        p.state = reinterpret_cast<float *>(a.ws + h.state());
        p.out16 = reinterpret_cast<uint16_t *>(a.ws + h.operand((i + 1) & 1));
        p.o = i + 1 == a.steps ? a.o : nullptr;
        p.ldo = a.ldo;
        p.otype = a.otype;
        p.x = h.wide() ? pl : st;
        p.xhop = h.wide() ? 2 * h.of_square() : 2 * h.of_state();
        p.w = h.wide() ? st : pl;
        p.whop = h.wide() ? 2 * h.of_state() : 2 * h.of_square();
        // from the left: the rows of P, and X across; from the right: X's rows, and P's, which are its columns
        p.inner = mp;
        e = h.wide() ? launch_tile<kAlong, kAcross, kApply>(p, s) : launch_tile<kAlong, kAlong, kApply>(p, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace isc
