// The experts' products (expert_linear.hip, expert_grad.hip): what the launches
// share, and the lists that a call's first launch makes of its route.
#pragma once

#include "tile_product.hpp"

namespace isc {

// Pairs p = t * slots + j by expert, as the products read them: made by
// expert_plan_kernel from a route's lists, with what lies outside of them taken out.
struct ExpertPlan {
    int32_t *tiles;   // the number of row tiles, then from [4] on four words each: expert, first place, rows, 0
    int32_t *pairs;   // P: the pair at each place of the experts' order, -1 where there is none
    int32_t *tokens;  // P: its token, -1 where there is none
};

struct ExpertArgs {
    int T, E, N, K, slots, type, shared;  // shared: a row of x for each token, not for each pair
    const void *x, *w;
    int64_t ldx, ldw;
    const int32_t *ids, *offsets, *order;
    const float *weights;
    ExpertPlan plan;
    int64_t pairs() const { return static_cast<int64_t>(T) * slots; }
};

struct ExpertLinearArgs {
    ExpertArgs a;
    void *y;
    int64_t ldy;
    int ytype, relu, combine;
    float *part;  // combine: P rows of fp32 sums, expert_ld() apart
};

struct ExpertBwdArgs {
    ExpertArgs a;
    const void *dy, *y;  // y: the rectified output, nullptr without a rectifier
    int64_t lddy, ldy;
    int combine;
    void *dx, *dw;        // each nullptr where it is not asked for
    float *dweights;
    int64_t lddx;
    void *masked;         // P rows of dy by expert: rectified or weighted, expert_ld() elements apart
    float *part, *dots;   // part: P rows of dx; dots: what each row's tiles give to dweights
};

// Leading dimension of rows in the workspace: 16-byte boundaries in every type.
inline int64_t expert_ld(int64_t cols) { return (cols + 7) / 8 * 8; }
// Rows of a tile of the experts' pairs, and the parts in which a row's dot products come.
int expert_tile_rows(int64_t pairs, int E, int type);
int expert_dots(int64_t pairs, int E, int K, int type);
size_t expert_plan_bytes(int64_t pairs, int E, int type);
ExpertPlan expert_plan_at(void *ws, int64_t pairs, int E, int type);

// Whether each of a call's launches has fewer threads than a launch may have.
bool expert_launches_fit(int64_t pairs, int E, int N, int K, int type);
// Where the parts of a gradient's workspace begin, and what all take.
struct ExpertBwdBytes {
    size_t masked, part, dots, all;
};
ExpertBwdBytes expert_bwd_bytes(int T, int E, int N, int K, int slots, int type, bool shared, bool relu, bool combine);

hipError_t launch_expert_plan(const ExpertArgs &a, void *empty, int64_t ld, int cols, int size, hipStream_t s);
// out[t] = the sum over a token's pairs of part's rows, weighted or not.
hipError_t launch_expert_sum(const ExpertArgs &a, const float *part, int cols, const float *weights, void *out,
                             int64_t ldo, int type, hipStream_t s);
hipError_t launch_expert_linear(const ExpertLinearArgs &a, hipStream_t s);
hipError_t launch_expert_bwd(const ExpertBwdArgs &a, hipStream_t s);

namespace tp {

// A product over rows by expert: out[pair] = sum over r of X(pair, r) W_e(j, r).
struct RowsArgs {
    ExpertPlan plan;
    Rows x, w;          // w: the first expert's
    int64_t expert;     // bytes from one expert's matrix to the next
    int listed;         // whether x.list is read by place; else places are x's rows
    int inner, cols;    // inner indices, columns of the result
    void *out;
    int64_t ldo;
    int otype, relu;
    const float *scale;  // of each pair's results, or nullptr
    const void *dotted;  // dots: each pair's results times this row, or nullptr
    int64_t lddot;
    int dot_slots;       // dotted has a row for every so many pairs
    float *dots;
    int ndots;
};

template <class TL>
__global__ __launch_bounds__(TL::kThreads) void expert_rows_kernel(const RowsArgs a) {
    using T = typename TL::T;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int across = (a.cols + TL::BJ - 1) / TL::BJ;
    const int total = a.plan.tiles[0] * across;
    if (static_cast<int>(blockIdx.x) >= total) return;
    const int id = of_xcd(blockIdx.x, total);
    const int4 tile = reinterpret_cast<const int4 *>(a.plan.tiles)[1 + id / across];
    const int e = __builtin_amdgcn_readfirstlane(tile.x), first = __builtin_amdgcn_readfirstlane(tile.y),
              rows = __builtin_amdgcn_readfirstlane(tile.z), j0 = id % across * TL::BJ;
    Rows x = a.x, w = a.w;
    if (a.listed)
        x.list += first;
    else
        x.base += first * x.stride;
    x.count = rows;
    w.base += e * a.expert;
    TL t;
    t.run(x, w, 0, j0, a.inner, rows, a.cols - j0, lds);
    float dot[TL::FI];
    t.each([&](int f, int i, int j, const f32x16 &sums) {
        const int p = i < rows ? a.plan.pairs[first + i] : -1;
        const int there = a.cols - j0 - j;
        f32x16 v = sums;
        if (a.dotted) {
            float d = 0.0f;
            if (p >= 0 && there > 0) {
                const auto *row = static_cast<const typename T::type *>(a.dotted) + p / a.dot_slots * a.lddot + j0 + j;
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float u[8];
                    load8<T>(u, row + 8 * q, there - 8 * q);
#pragma unroll
                    for (int n = 0; n < 8; ++n) d = fmaf(n + 8 * q < there ? v[8 * q + n] : 0.0f, u[n], d);
                }
            }
            d += __shfl_xor(d, 32);
            dot[f] = j % (TL::BJ / TL::WJ) < 32 ? d : dot[f] + d;
            if (j % (TL::BJ / TL::WJ) >= TL::BJ / TL::WJ - 32 && (threadIdx.x & 63) < 32 && p >= 0)
                a.dots[static_cast<int64_t>(p) * a.ndots + j0 / TL::BJ * TL::WJ + TL::part_j() / (TL::BJ / TL::WJ)] = dot[f];
        }
        if (p < 0 || there <= 0) return;
        if (a.scale) {
            const float s = a.scale[p];
#pragma unroll
            for (int n = 0; n < 16; ++n) v[n] *= s;
        }
        if (a.relu) {
#pragma unroll
            for (int n = 0; n < 16; ++n) v[n] = v[n] < 0.0f ? 0.0f : v[n];  // a NaN stays
        }
        const int64_t at = p * a.ldo + j0 + j;
        if (a.otype == ISC_F32)
            store16<F32>(static_cast<float *>(a.out) + at, v, there);
        else if (a.otype == ISC_BF16)
            store16<BF16>(static_cast<uint16_t *>(a.out) + at, v, there);
        else
            store16<F16>(static_cast<uint16_t *>(a.out) + at, v, there);
    });
}

// Whether a side's rows can go into LDS by direct loads.
inline bool direct_rows(const void *p, int64_t ld, int width, int size) {
    return size == 2 && reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && width % 8 == 0;
}

template <class TL>
hipError_t launch_rows(const RowsArgs &a, int64_t pairs, int E, hipStream_t s) {
    if (hipError_t e = allow_lds(expert_rows_kernel<TL>, TL::kLds); e != hipSuccess) return e;
    const int64_t tiles = pairs / TL::BI + (pairs < E ? pairs : E);  // as many as there can be
    const int64_t grid = tiles * ((a.cols + TL::BJ - 1) / TL::BJ);
    hipLaunchKernelGGL(expert_rows_kernel<TL>, dim3(static_cast<unsigned>(grid)), dim3(TL::kThreads), TL::kLds, s, a);
    return hipGetLastError();
}

// The tiles of 16- and 32-bit rows: few rows, or many.
template <class T, bool DIRECT, Side WS>
hipError_t launch_rows_of(const RowsArgs &a, int64_t pairs, int E, int rows, hipStream_t s) {
    if constexpr (std::is_same_v<T, F32>) {
        if (rows == 64) return launch_rows<Tile<T, false, kAlong, WS, 64, 128, 1, 4>>(a, pairs, E, s);
        return launch_rows<Tile<T, false, kAlong, WS, 128, 128, 2, 2>>(a, pairs, E, s);
    } else {
        if (rows == 32) return launch_rows<Tile<T, DIRECT, kAlong, WS, 32, 128, 1, 4>>(a, pairs, E, s);
        if (rows == 256) return launch_rows<Tile<T, DIRECT, kAlong, WS, 256, 256, 2, 4>>(a, pairs, E, s);
        return launch_rows<Tile<T, DIRECT, kAlong, WS, 128, 128, 2, 2>>(a, pairs, E, s);
    }
}
template <Side WS>
hipError_t launch_rows_by(const RowsArgs &a, int type, bool direct, int64_t pairs, int E, hipStream_t s) {
    const int rows = expert_tile_rows(pairs, E, type);
    if (type == ISC_F32) return launch_rows_of<F32, false, WS>(a, pairs, E, rows, s);
    if (type == ISC_BF16)
        return direct ? launch_rows_of<BF16, true, WS>(a, pairs, E, rows, s)
                      : launch_rows_of<BF16, false, WS>(a, pairs, E, rows, s);
    return direct ? launch_rows_of<F16, true, WS>(a, pairs, E, rows, s)
                  : launch_rows_of<F16, false, WS>(a, pairs, E, rows, s);
}

}  // namespace tp
}  // namespace isc
