// Orthogonalising updates (isc_orthogonalize): X = G / (|G| + eps), |G| the
// Frobenius norm, then some steps of
//   X <- a X + (b A + c A^2) X,  A = X X^T     (A = X^T X from the right, where G is tall)
// an odd polynomial of X's singular values that leaves its singular vectors as
// they are and brings the values towards one.
//
// What is held how.  What a step adds to a small singular direction is small beside the
// large ones, and every later step magnifies an error there as it does the direction
// (3.4^5 = 480 in all): a state of one fp16 value gives a result 4 % off where noise of
// 0.01 lies over 16 directions (704 x 2048; bf16 34 %).  The state X is held in 32 bits,
// as the fp16 value that the products take and what that leaves, in fp16 as well: 22 bits
// in all, read and written with 8 bytes an element and step where fp32 beside the operand
// takes 10.  The operands of the products, X's first part, A and b A + c A^2, are fp16,
// whose errors stay where the operand is one factor among fp32 sums: 3.3e-4 of the same
// result, 1.5e-3 on noise alone, its rounding to bf16 1.7e-3.  (Where a side is at most 64 the
// operands are in two parts as well: orth_small.hip.)  Operands are scaled by 2^6
// on their way to fp16, which keeps entries of 2^-14 normal and any that the coefficients'
// check lets through finite; what they leave by 2^11 more.
//
// A and b A + c A^2 are symmetric: tiles on and below the diagonal are computed,
// the others are their mirror images.  All matrices of a stack share each launch:
// three products a step.  What bounds it: the matrix cores.
#include "orthogonalize.hpp"

#include "tile_product.hpp"

namespace isc {
namespace {

using namespace tp;

constexpr float kUp = kOrthUp, kLow = kOrthLow;

struct OrthProduct {
    OrthShape s;
    Rows x, w;              // the first matrix's
    int64_t xhop, whop;     // bytes to the next one's
    int inner, rows, cols;
    const uint16_t *from;   // A, where b A is added; the state's operand
    uint16_t *to;           // A, b A + c A^2, or the next state's operand
    uint16_t *low;          // what the state's operand leaves
    const void *g;          // the first step's state is G, scaled
    int64_t ldg;
    int type;
    const double *inverse;  // of the norms
    void *o;                // the last step's results
    int64_t ldo;
    int otype;
    float a, b, c;
    int parts;              // of A's sums, whose fp32 results go to `partial`
    float *partial;
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

// The first state's operand; the first step takes the state itself from G.  Both scale in
// fp64: the inverse of a small norm may be beyond fp32.
template <class T>
__global__ __launch_bounds__(256) void orth_scale_kernel(const OrthArgs a) {
    const OrthShape &s = a.s;
    const int64_t row0 = static_cast<int64_t>(blockIdx.y) * s.M;
    __shared__ double sums[256];
    const double by = orth_inverse_norm(reinterpret_cast<const double *>(a.ws), blockIdx.y, s.blocks(), a.eps, sums);
    if (blockIdx.x == 0 && threadIdx.x == 0) reinterpret_cast<double *>(a.ws + s.inverse())[blockIdx.y] = by;
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
            v[q] = c + q < s.N ? static_cast<float>(static_cast<double>(v[q]) * by) * kUp : 0.0f;
        store8<F16>(operand + r * s.np() + c, v, 8);
    }
}

enum Product { kGram, kPoly, kApply };

template <class TL, Product WHAT>
__global__ __launch_bounds__(TL::kThreads) void orth_product_kernel(const OrthProduct p, int total) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int down = (p.rows + TL::BI - 1) / TL::BI, across = (p.cols + TL::BJ - 1) / TL::BJ;
    struct Job {
        int n, i0, j0, part, inner;
    } job, next;
    struct Beside {  // the state's two parts, or G's values
        Raw8<F16> one, other;
    };
    TL t;
    const auto start = [&](int at) {
        int id = of_xcd(at, total), ti, tj, inner = p.inner;
        Job j;
        j.part = 0;
        if constexpr (WHAT == kApply) {
            j.n = id / (down * across);
            ti = id / across % down;
            tj = id % across;
        } else {
            const int half = down * (down + 1) / 2;
            if (WHAT == kGram) {
                j.part = id % p.parts;
                id /= p.parts;
            }
            j.n = id / half;
            id %= half;  // ti (ti + 1) / 2 + tj
            ti = static_cast<int>((__builtin_sqrtf(8.0f * id + 1.0f) - 1.0f) * 0.5f);
            if (ti * (ti + 1) / 2 > id) --ti;
            if ((ti + 1) * (ti + 2) / 2 <= id) ++ti;
            tj = id - ti * (ti + 1) / 2;
        }
        j.i0 = ti * TL::BI;
        j.j0 = tj * TL::BJ;
        Rows x = p.x, w = p.w;
        x.base += j.n * p.xhop;
        w.base += j.n * p.whop;
        if (WHAT == kGram && p.parts > 1) {  // a range of whole stages of the inner indices
            const int stages = (p.inner + TL::BK - 1) / TL::BK, from = stages * j.part / p.parts * TL::BK;
            const int to = stages * (j.part + 1) / p.parts * TL::BK;
            inner = (to < p.inner ? to : p.inner) - from;
            if (TL::kXAcross) {
                x.base += from * x.stride;
                w.base += from * w.stride;
                x.count = w.count = inner;
            } else {
                x.base += int64_t{2} * from;
                w.base += int64_t{2} * from;
                x.width = w.width = inner;
            }
        }
        j.inner = inner;
        t.start(x, w, j.i0, j.j0, inner, lds);
        return j;
    };
    int at = blockIdx.x;
    job = start(at);
    for (bool landed = false;; landed = true) {
        t.sums(job.inner, p.rows - job.i0, p.cols - job.j0, landed, lds);
        at += gridDim.x;
        if (at < total) next = start(at);
        if constexpr (WHAT == kApply) {
            const int np = p.s.np();
            const int64_t first = job.n * p.s.of_state();
            const double by = p.g ? p.inverse[job.n] : 0.0;
            t.template each<false>(
                lds,
                [&](int i, int j) {
                    Beside b = {};
                    const int row = job.i0 + i, col = job.j0 + j;
                    if (row >= p.rows || col >= p.cols) return b;
                    if (p.g) {
                        const int64_t place = (static_cast<int64_t>(job.n) * p.rows + row) * p.ldg + col;
                        if (p.type == ISC_F32) {
                            Raw8<F32> g;
                            g.load(static_cast<const float *>(p.g) + place, p.cols - col);
                            b.one.a = g.a;
                            b.other.a = g.b;
                        } else {
                            b.one.load(static_cast<const uint16_t *>(p.g) + place, p.cols - col);
                        }
                    } else {
                        const int64_t place = first + static_cast<int64_t>(row) * np + col;
                        b.one.load(p.from + place, 8);
                        b.other.load(p.low + place, 8);
                    }
                    return b;
                },
                [&](int i, int j, const float (&sums)[8], const Beside &beside) {
                    const int row = job.i0 + i, col = job.j0 + j;
                    if (row >= p.rows || col >= p.cols) return;
                    const int64_t place = first + static_cast<int64_t>(row) * np + col;
                    float x[8], v[8];
                    if (p.g) {
                        if (p.type == ISC_F32)
                            Raw8<F32>{beside.one.a, beside.other.a}.widen(x);
                        else if (p.type == ISC_BF16)
                            Raw8<BF16>{beside.one.a, {}}.widen(x);
                        else
                            beside.one.widen(x);
#pragma unroll
                        for (int k = 0; k < 8; ++k) x[k] = static_cast<float>(static_cast<double>(x[k]) * by) * kUp;
                    } else {
                        float low[8];
                        beside.one.widen(x);
                        beside.other.widen(low);
#pragma unroll
                        for (int k = 0; k < 8; ++k) x[k] = fmaf(low[k], 1.0f / kLow, x[k]);
                    }
                    // x and what becomes of it are 2^6 times the state, the sums 2^12 times theirs;
                    // behind the last column the operands' zeros made zeros, or another column's sums
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        v[k] = col + k < p.cols ? fmaf(p.a, x[k], sums[k] * (1.0f / kUp)) : 0.0f;
                    if (p.o) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] *= 1.0f / kUp;
                        store8_as(p.o, (static_cast<int64_t>(job.n) * p.rows + row) * p.ldo + col, v, p.cols - col,
                                  p.otype);
                        return;
                    }
                    float low[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) low[k] = (v[k] - F16::widen(F16::narrow(v[k]))) * kLow;
                    store8<F16>(p.to + place, v, 8);
                    store8<F16>(p.low + place, low, 8);
                },
                [](int, int, const float (&)[8]) {});
        } else {
            const int m = p.rows, mp = p.s.mp();
            const int64_t first = job.n * p.s.of_square();
            const bool mirror = job.i0 != job.j0;
            const auto store = [&](int row, int col, const float (&v)[8]) {
                const int64_t place = first + static_cast<int64_t>(row) * mp + col;
                if (WHAT == kGram && p.parts > 1)
                    store8<F32>(p.partial + job.part * p.s.B * p.s.of_square() + place, v, 8);
                else
                    store8<F16>(p.to + place, v, 8);
            };
            t.template each<true>(
                lds,
                [&](int i, int j) {
                    Raw8<F16> u = {};
                    const int row = job.i0 + i, col = job.j0 + j;
                    if (WHAT == kPoly && row < m && col < mp) u.load(p.from + first + static_cast<int64_t>(row) * mp + col, 8);
                    return u;
                },
                // A, or b A + c A^2, zeros behind the last column
                [&](int i, int j, float (&v)[8], const Raw8<F16> &beside) {
                    const int row = job.i0 + i, col = job.j0 + j;
                    float u[8];
                    beside.widen(u);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        v[k] *= 1.0f / kUp;
                        if (WHAT == kPoly) v[k] = fmaf(p.b, u[k], p.c * v[k]);
                        v[k] = row < m && col + k < m ? v[k] : 0.0f;
                    }
                    if (row < m && col < mp) store(row, col, v);
                },
                [&](int j, int i, const float (&v)[8]) {
                    const int row = job.j0 + j, col = job.i0 + i;
                    if (mirror && row < m && col < mp) store(row, col, v);
                });
        }
        if (at >= total) return;
        job = next;
    }
}

// A from the parts of its sums, in their order.
__global__ __launch_bounds__(256) void orth_join_kernel(const float *partial, int parts, int64_t n, uint16_t *to) {
    const int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8;
    if (i >= n) return;  // n is a multiple of 8
    float sum[8] = {};
#pragma unroll 4
    for (int q = 0; q < parts; ++q) {
        float v[8];
        load8<F32>(v, partial + q * n + i, 8);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] += v[k];
    }
    store8<F16>(to + i, sum, 8);
}

template <class TL, Product WHAT>
hipError_t launch_product(const OrthProduct &p, hipStream_t s) {
    if (hipError_t e = (allow_lds<orth_product_kernel<TL, WHAT>>(TL::kLds)); e != hipSuccess) return e;
    const int64_t down = (p.rows + TL::BI - 1) / TL::BI, across = (p.cols + TL::BJ - 1) / TL::BJ;
    const int64_t total = p.s.B * (WHAT == kApply ? down * across : down * (down + 1) / 2 * (WHAT == kGram ? p.parts : 1));
    hipLaunchKernelGGL((orth_product_kernel<TL, WHAT>),
                       dim3(static_cast<unsigned>(total < kResident<TL> ? total : kResident<TL>)), dim3(TL::kThreads),
                       TL::kLds, s, p, static_cast<int>(total));
    return hipGetLastError();
}

template <Side XS, Side WS, Product WHAT>
hipError_t launch_tile(const OrthProduct &p, hipStream_t s) {
    const auto tiles = [&](int side) {
        const int64_t down = (p.rows + side - 1) / side, across = (p.cols + side - 1) / side;
        return p.s.B * (WHAT == kApply ? down * across : down * (down + 1) / 2);
    };
    const int side = WHAT == kGram && p.parts > 1 ? 64 : tile_side(tiles(256), tiles(128), false);
    if (side == 256) return launch_product<Tile<F16, true, XS, WS, 256, 256, 2, 4>, WHAT>(p, s);
    if (side == 128) return launch_product<Tile<F16, true, XS, WS, 128, 128, 2, 2>, WHAT>(p, s);
    if (hipError_t e = launch_product<Tile<F16, true, XS, WS, 64, 64, 2, 2>, WHAT>(p, s); e != hipSuccess) return e;
    if (WHAT != kGram || p.parts == 1) return hipSuccess;
    const int64_t n = p.s.B * p.s.of_square();
    hipLaunchKernelGGL(orth_join_kernel, dim3(static_cast<unsigned>((n / 8 + 255) / 256)), dim3(256), 0, s, p.partial,
                       p.parts, n, p.to);
    return hipGetLastError();
}

dim3 norm_grid(const OrthShape &s) { return dim3(static_cast<unsigned>(s.blocks()), static_cast<unsigned>(s.B)); }

template <class T>
hipError_t launch_scale(const OrthArgs &a, hipStream_t s) {
    hipLaunchKernelGGL(orth_scale_kernel<T>, norm_grid(a.s), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_orth_norm(const OrthArgs &a, hipStream_t s) {
    if (a.type == ISC_F32)
        hipLaunchKernelGGL(orth_norm_kernel<F32>, norm_grid(a.s), dim3(256), 0, s, a);
    else if (a.type == ISC_BF16)
        hipLaunchKernelGGL(orth_norm_kernel<BF16>, norm_grid(a.s), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL(orth_norm_kernel<F16>, norm_grid(a.s), dim3(256), 0, s, a);
    return hipGetLastError();
}

bool orth_launches_fit(const OrthShape &s) {
    const int64_t down = (s.M + 63) / 64, across = (s.N + 63) / 64, m = (s.m() + 63) / 64;
    const int64_t most = down * across > m * (m + 1) / 2 ? down * across : m * (m + 1) / 2;
    return s.B * most < int64_t{1} << 31;
}

hipError_t launch_orthogonalize(const OrthArgs &a, hipStream_t s) {
    const OrthShape &h = a.s;
    hipError_t e = launch_orth_norm(a, s);
    if (e != hipSuccess) return e;
    if (h.small()) return launch_orth_small(a, s);
    e = a.type == ISC_F32    ? launch_scale<F32>(a, s)
        : a.type == ISC_BF16 ? launch_scale<BF16>(a, s)
                             : launch_scale<F16>(a, s);
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
        p.to = square;
        p.from = square;
        p.inner = h.wide() ? np : h.M;
        p.parts = h.parts();
        p.partial = reinterpret_cast<float *>(a.ws + h.partial());
        e = h.wide() ? launch_tile<kAlong, kAlong, kGram>(p, s) : launch_tile<kAcross, kAcross, kGram>(p, s);
        if (e != hipSuccess) return e;
        const Rows sq{reinterpret_cast<const char *>(square), int64_t{2} * mp, nullptr, m, mp};
        p.x = p.w = sq;
        p.xhop = p.whop = 2 * h.of_square();
        p.inner = mp;
        p.to = poly;
        if ((e = launch_tile<kAlong, kAlong, kPoly>(p, s)) != hipSuccess) return e;
        const Rows pl{reinterpret_cast<const char *>(poly), int64_t{2} * mp, nullptr, m, mp};
        const Rows st{x, int64_t{2} * np, nullptr, h.M, np};
        p.rows = h.M;
        p.cols = h.N;
        p.from = reinterpret_cast<const uint16_t *>(x);
        p.to = reinterpret_cast<uint16_t *>(a.ws + h.operand((i + 1) & 1));
        p.low = reinterpret_cast<uint16_t *>(a.ws + h.low());
        if (i == 0) {
            p.g = a.g;
            p.ldg = a.ldg;
            p.type = a.type;
            p.inverse = reinterpret_cast<const double *>(a.ws + h.inverse());
        }
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
