// The gradients of the experts' products (isc_expert_linear_bwd).
//
// With d[p] the gradient that reaches pair p's product (dy masked where the
// rectified output is 0, or its token's dy for a sum under weights):
//   dx[p] = s w[e]^T d[p], s the pair's weight or 1; summed over a token's slots
//     where they share a row of x.  A product over N whose matrix is stored with N
//     across its rows: the transposing LDS read turns it over.
//   dweights[p] = (w[e]^T d[p]) . x[p]: from dx's own sums, before their weight, so
//     the product w x is not made again; each tile of columns gives a part.
//   dw[e] = sum over e's pairs of s d[p] x[p]^T: as many terms as e has pairs, and
//     both operands have them across their rows.
// Masked or weighted gradients are written once, in their own type (a
// weight times a gradient is rounded there: half a unit in the last place of each
// term, which leaves of a sum what the sum's own rounding is), since the product
// that reads them would do it for every tile.
#include "expert.hpp"

namespace isc {
namespace {

using namespace tp;

// masked[i] = the gradient of the product of the pair at place i, 0 where an expert's place has
// no pair.  In the places' order, so that the products read consecutive rows.
template <class T>
__global__ __launch_bounds__(256) void expert_mask_kernel(const ExpertBwdArgs b, int64_t ld) {
    const ExpertArgs &a = b.a;
    using V = typename T::type;
    const int groups = static_cast<int>(ld / 8);
    const int64_t all = static_cast<int64_t>(a.T) * a.slots * groups, hop = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; n < all; n += hop) {
        const int64_t i = n / groups, p = a.plan.pairs[i];
        const int c = static_cast<int>(n - i * groups) * 8;
        const bool there = p >= 0;
        if (!there && i >= a.offsets[a.E]) continue;
        float v[8] = {};
        if (there) {
            load8<T>(v, static_cast<const V *>(b.dy) + (b.combine ? p / a.slots : p) * b.lddy + c, a.N - c);
            if (b.y) {
                float y[8];
                load8<T>(y, static_cast<const V *>(b.y) + p * b.ldy + c, a.N - c);
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = y[q] <= 0.0f ? 0.0f : v[q];
            }
            if (b.combine) {
                const float w = a.weights[p];
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = c + q < a.N ? v[q] * w : 0.0f;
            }
        }
        store8<T>(static_cast<V *>(b.masked) + i * ld + c, v, 8);
    }
}

// dweights[p] from its tiles' parts, in their order.
__global__ __launch_bounds__(256) void expert_dots_kernel(const ExpertArgs a, const float *dots, int n, float *out) {
    const int64_t p = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int P = a.T * a.slots;
    if (p >= P) return;
    float sum = 0.0f;
    if (expert_listed(a.plan, P, static_cast<int>(p)))
        for (int i = 0; i < n; ++i) sum += dots[p * n + i];
    out[p] = sum;
}

struct DwArgs {
    const int32_t *offsets, *by_size;
    Rows d, x;  // listed by place, or d's in the places' order
    int P, N, K;
    void *dw;
    int nexp;
};

template <class TL>
__global__ __launch_bounds__(TL::kThreads) void expert_dw_kernel(const DwArgs a, int total) {
    using T = typename TL::T;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int down = (a.N + TL::BI - 1) / TL::BI, across = (a.K + TL::BJ - 1) / TL::BJ;
    struct Job {
        int e, i0, j0, inner;
    } job, next;
    TL t;
    const auto start = [&](int n) {
        const int id = of_xcd(n, total);
        Job j{a.by_size ? a.by_size[id / (down * across)] : id / (down * across), id / across % down * TL::BI, id % across * TL::BJ, 0};
        const int lo = a.offsets[j.e], hi = a.offsets[j.e + 1];
        const int first = lo < 0 ? 0 : lo > a.P ? a.P : lo, end = hi > a.P ? a.P : hi;
        Rows d = a.d, x = a.x;
        d.count = x.count = j.inner = end > first ? end - first : 0;
        if (d.list)
            d.list += first;
        else
            d.base += first * d.stride;
        x.list += first;
        t.start(d, x, j.i0, j.j0, j.inner, lds);
        return j;
    };
    int n = blockIdx.x;
    job = start(n);
    for (bool landed = false;; landed = true) {
        t.sums(job.inner, a.N - job.i0, a.K - job.j0, landed, lds);
        n += gridDim.x;
        if (n < total) next = start(n);
        auto *dw = static_cast<typename T::type *>(a.dw) + static_cast<int64_t>(job.e) * a.N * a.K;
        t.template each<false>(
            lds,
            [](int, int) { return 0; },
            [&](int i, int j, const float (&v)[8], int) {
                if (job.i0 + i < a.N && job.j0 + j < a.K)
                    store8<T>(dw + static_cast<int64_t>(job.i0 + i) * a.K + job.j0 + j, v, a.K - job.j0 - j);
            },
            [](int, int, const float (&)[8]) {});
        if (n >= total) return;
        job = next;
    }
}

// Without tokens every weight's gradient is 0, and there are no lists to read.
__global__ __launch_bounds__(256) void expert_zero_kernel(uint16_t *p, int64_t n) {
    const int64_t hop = static_cast<int64_t>(gridDim.x) * 2048;
    for (int64_t i = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8; i < n; i += hop) {
        if (n - i >= 8)
            store_any(p + i, make_uint4(0, 0, 0, 0));
        else
            for (int64_t q = i; q < n; ++q) p[q] = 0;
    }
}
hipError_t launch_zero_dw(const ExpertBwdArgs &b, hipStream_t s) {
    const int64_t n = static_cast<int64_t>(b.a.E) * b.a.N * b.a.K * (b.a.type == ISC_F32 ? 2 : 1);
    const int64_t blocks = (n + 2047) / 2048;
    hipLaunchKernelGGL(expert_zero_kernel, dim3(static_cast<unsigned>(blocks < 8192 ? blocks : 8192)), dim3(256), 0, s,
                       static_cast<uint16_t *>(b.dw), n);
    return hipGetLastError();
}

template <class TL>
hipError_t launch_dw(const DwArgs &a, hipStream_t s) {
    if (hipError_t e = allow_lds<expert_dw_kernel<TL>>(TL::kLds); e != hipSuccess) return e;
    const int64_t grid = static_cast<int64_t>((a.N + TL::BI - 1) / TL::BI) * ((a.K + TL::BJ - 1) / TL::BJ) * a.nexp;
    hipLaunchKernelGGL(expert_dw_kernel<TL>, dim3(static_cast<unsigned>(grid < kResident<TL> ? grid : kResident<TL>)),
                       dim3(TL::kThreads), TL::kLds, s, a, static_cast<int>(grid));
    return hipGetLastError();
}
template <class T, bool DIRECT>
hipError_t launch_dw_of(const DwArgs &a, hipStream_t s) {
    const auto tiles = [&](int side) {
        return static_cast<int64_t>(a.nexp) * ((a.N + side - 1) / side) * ((a.K + side - 1) / side);
    };
    const int side = tile_side(DIRECT ? tiles(256) : 0, tiles(128), std::is_same_v<T, F32>);
    if constexpr (DIRECT)
        if (side == 256)
            return a.d.list ? launch_dw<Tile<T, true, kAcross, kAcross, 256, 256, 2, 4, 3>>(a, s)
                            : launch_dw<Tile<T, true, kAcross, kAcross, 256, 256, 2, 4, 2>>(a, s);
    if (side == 128) return launch_dw<Tile<T, DIRECT, kAcross, kAcross, 128, 128, 2, kWavesOf128<T>, 3>>(a, s);
    return launch_dw<Tile<T, DIRECT, kAcross, kAcross, 64, 64, 2, 2, 3, kInner64<DIRECT>>>(a, s);
}

template <class T>
hipError_t launch_mask(const ExpertBwdArgs &b, hipStream_t s) {
    const int64_t ld = expert_ld(b.a.N), blocks = (b.a.pairs() * (ld / 8) + 255) / 256;
    hipLaunchKernelGGL(expert_mask_kernel<T>, dim3(static_cast<unsigned>(blocks < 16384 ? blocks : 16384)), dim3(256),
                       0, s, b, ld);
    return hipGetLastError();
}

}  // namespace

int expert_dots(int64_t pairs, int E, int K, int type, bool direct) {
    const int cols = expert_tile_rows(pairs, E, K, type, direct) >= 128 && type != ISC_F32 ? 64 : 32;  // of a wavefront
    return (K + cols - 1) / cols;
}

ExpertBwdBytes expert_bwd_bytes(int T, int E, int N, int K, int slots, int type, bool shared, bool relu, bool combine) {
    const int64_t pairs = static_cast<int64_t>(T) * slots;
    const auto round = [](int64_t n) { return static_cast<size_t>((n + 255) / 256 * 256); };
    ExpertBwdBytes b;
    b.masked = expert_plan_bytes(pairs, E, type);
    b.part = b.masked + (relu || combine ? round(pairs * expert_ld(N) * (type == ISC_F32 ? 4 : 2)) : 0);
    // a call without dx has its rows there too
    b.dots = b.part + (combine || (shared && slots > 1) ? round(pairs * expert_ld(K) * 4) : 0);
    b.all = b.dots + (combine ? round(pairs * ((K + 31) / 32) * 4) : 0);
    return b;
}

hipError_t launch_expert_bwd(const ExpertBwdArgs &b, hipStream_t s) {
    const ExpertArgs &a = b.a;
    const int size = a.type == ISC_F32 ? 4 : 2;
    const bool sum = a.shared && a.slots > 1;
    if (a.T == 0) return launch_zero_dw(b, s);
    const int64_t ldm = expert_ld(a.N);
    const bool aligned_dy = direct_rows(b.dy, b.lddy, a.N, size), aligned_masked = direct_rows(b.masked, ldm, a.N, size);
    const bool direct = (b.y ? aligned_masked : aligned_dy) && direct_rows(a.w, a.ldw, a.K, size);
    // where every workgroup has tiles of several experts
    const bool by_size = b.dw && static_cast<int64_t>(a.E) * ((a.N + 255) / 256) * ((a.K + 255) / 256) > 512;
    hipError_t e = launch_expert_plan(a, expert_tile_rows(a.pairs(), a.E, a.K, a.type, direct), by_size, s);
    if (e != hipSuccess) return e;
    // a sum's dx takes the gradient as it is (its own sums are weighted), a rectifier's takes it masked
    const bool masks = b.y || (b.combine && b.dw);
    if (masks) {
        e = a.type == ISC_F32 ? launch_mask<F32>(b, s) : a.type == ISC_BF16 ? launch_mask<BF16>(b, s) : launch_mask<F16>(b, s);
        if (e != hipSuccess) return e;
    }
    const Rows masked{static_cast<const char *>(b.masked), ldm * size, nullptr, 0, a.N};
    const Rows given{static_cast<const char *>(b.dy), b.lddy * size, b.combine ? a.plan.tokens : a.plan.pairs, 0, a.N};
    if (b.dx || b.dweights) {
        RowsArgs r = rows_of(a, !b.dx ? kLeave : sum ? kWithExpert : kAll);
        r.x = b.y ? masked : given;
        r.w = {static_cast<const char *>(a.w), a.ldw * size, nullptr, a.N, a.K};
        r.expert = a.N * a.ldw * size;
        r.inner = a.N;
        r.cols = a.K;
        r.out = sum || !b.dx ? b.part : b.dx;
        r.ldo = sum || !b.dx ? expert_ld(a.K) : b.lddx;
        r.otype = sum || !b.dx ? ISC_F32 : a.type;
        r.scale = b.combine ? a.weights : nullptr;
        if (b.dweights) {
            r.dotted = a.x;
            r.lddot = a.ldx;
            r.dot_slots = a.shared ? a.slots : 1;
            r.dots = b.dots;
            r.ndots = expert_dots(a.pairs(), a.E, a.K, a.type, direct);
        }
        e = launch_rows_by<kAcross>(r, a.type, direct, a.pairs(), a.E, s);
        if (e != hipSuccess) return e;
        if (sum && b.dx) {
            e = launch_expert_sum(a, b.part, a.K, nullptr, b.dx, b.lddx, a.type, s);
            if (e != hipSuccess) return e;
        }
        if (b.dweights) {
            hipLaunchKernelGGL(expert_dots_kernel, dim3(static_cast<unsigned>((a.pairs() + 255) / 256)), dim3(256), 0, s, a,
                               b.dots, r.ndots, b.dweights);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    if (!b.dw) return hipSuccess;
    const DwArgs d{a.offsets, by_size ? a.plan.by_size : nullptr,
                   masks ? masked : given,
                   {static_cast<const char *>(a.x), a.ldx * size, a.shared ? a.plan.tokens : a.plan.pairs, 0, a.K},
                   static_cast<int>(a.pairs()), a.N, a.K, b.dw, a.E};
    const bool direct_x = (masks ? aligned_masked : aligned_dy) && direct_rows(a.x, a.ldx, a.K, size);
    if (a.type == ISC_F32) return launch_dw_of<F32, false>(d, s);
    if (a.type == ISC_BF16) return direct_x ? launch_dw_of<BF16, true>(d, s) : launch_dw_of<BF16, false>(d, s);
    return direct_x ? launch_dw_of<F16, true>(d, s) : launch_dw_of<F16, false>(d, s);
}

}  // namespace isc
