// The experts' products (expert_linear.hip, expert_grad.hip): what the launches
// share, and the lists that a call's first launch makes of its route.
#pragma once

#include "tile_product.hpp"

namespace isc {

// Pairs p = t * slots + j by expert, as the products read them: made by
// expert_plan_kernel from a route's lists, with what lies outside of them taken out.
struct ExpertPlan {
    int32_t *tiles;   // the number of row tiles, then from [4] on four words each: expert, first place, rows, 0
    int32_t *pairs;   // P: the pair at each place of the experts' order, -1 where it holds none of its expert's
    int32_t *tokens;  // P: its token, -1 where there is none
    int32_t *places;  // P: a place that holds the pair; anything where none does (expert_listed)
    int32_t *by_size; // E: the experts in the order of weight gradients' tiles (expert_by_size)
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
    void *masked;         // P rows of dy, rectified or weighted, in the places' order, expert_ld() elements apart
    float *part, *dots;   // part: P rows of dx; dots: what each row's tiles give to dweights
};

// Leading dimension of rows in the workspace: 16-byte boundaries in every type.
inline int64_t expert_ld(int64_t cols) { return (cols + 7) / 8 * 8; }
// Rows of a tile of the experts' pairs for a product with `cols` columns (direct: of operands
// that go into LDS by direct loads), and the parts in which a row's dot products come.
int expert_tile_rows(int64_t pairs, int E, int cols, int type, bool direct);
int expert_dots(int64_t pairs, int E, int K, int type, bool direct);
size_t expert_plan_bytes(int64_t pairs, int E, int type);
ExpertPlan expert_plan_at(void *ws, int64_t pairs, int E, int type);

// Whether each of a call's launches has fewer threads than a launch may have.
bool expert_launches_fit(int64_t pairs, int E, int N, int K, int type);
// Where the parts of a gradient's workspace begin, and what all take.
struct ExpertBwdBytes {
    size_t masked, part, dots, all;
};
ExpertBwdBytes expert_bwd_bytes(int T, int E, int N, int K, int slots, int type, bool shared, bool relu, bool combine);

// Tiles of `rows` rows.  by_size: whether the experts' order is made too.
hipError_t launch_expert_plan(const ExpertArgs &a, int rows, bool by_size, hipStream_t s);
// out[t] = the sum over a token's pairs of part's rows, weighted or not.
hipError_t launch_expert_sum(const ExpertArgs &a, const float *part, int cols, const float *weights, void *out,
                             int64_t ldo, int type, hipStream_t s);
hipError_t launch_expert_linear(const ExpertLinearArgs &a, hipStream_t s);
// The same for few pairs (expert_few.hip): one launch, and a sum's; no plan.
bool expert_few(int64_t pairs, int E, int type);
hipError_t launch_expert_few(const ExpertLinearArgs &a, hipStream_t s);
hipError_t launch_expert_bwd(const ExpertBwdArgs &a, hipStream_t s);

#if defined(__HIPCC__)
// Whether a place of its expert's holds pair p of P.  Nothing clears `places`, where a pair that
// no place holds has what was in the workspace: the place that it names does not hold it.
__device__ __forceinline__ bool expert_listed(const ExpertPlan &plan, int P, int p) {
    const int i = plan.places[p];
    return static_cast<unsigned>(i) < static_cast<unsigned>(P) && plan.pairs[i] == p;
}
#endif

namespace tp {

// Which rows of the result become 0 of those that no place lists: none, those of pairs that
// have an expert (the others are not read), or all.
enum Unlisted { kLeave, kWithExpert, kAll };

// A product over rows by expert: out[pair] = sum over r of X(pair, r) W_e(j, r).
struct RowsArgs {
    ExpertPlan plan;
    Unlisted unlisted;
    const int32_t *ids;
    int P, E;
    Rows x, w;          // x by the list of places, or its rows in their order; w: the first expert's
    int64_t expert;     // bytes from one expert's matrix to the next
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

// The rows of pairs that no place lists, 64 pairs a wavefront in turn.
template <int WAVES>
__device__ __forceinline__ void clear_unlisted(const RowsArgs &a) {
    if (a.unlisted == kLeave) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int size = a.otype == ISC_F32 ? 4 : 2, bytes = a.cols * size, hop = gridDim.x * WAVES;
    for (int first = (wave * gridDim.x + blockIdx.x) * 64; first < a.P; first += hop * 64) {
        const int p = first + lane;
        const bool none = p < a.P && !expert_listed(a.plan, a.P, p) &&
                          (a.unlisted == kAll || static_cast<unsigned>(a.ids[p]) < static_cast<unsigned>(a.E));
        uint64_t mask = __ballot(none);
        while (mask) {
            char *row = static_cast<char *>(a.out) +
                        (first + __ffsll(static_cast<unsigned long long>(mask)) - 1) * a.ldo * size;
            mask &= mask - 1;
            for (int b = lane * 16; b < bytes; b += 1024) {
                if (b + 16 <= bytes)
                    store_any(row + b, make_uint4(0, 0, 0, 0));
                else
                    for (int c = b; c < bytes; c += 2) store_any(row + c, static_cast<uint16_t>(0));
            }
        }
    }
}

template <class TL>
__global__ __launch_bounds__(TL::kThreads) void expert_rows_kernel(const RowsArgs a) {
    using T = typename TL::T;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int across = (a.cols + TL::BJ - 1) / TL::BJ;
    const int total = a.plan.tiles[0] * across;
    struct Job {
        int first, rows, j0;
    } job, next;
    struct Beside {
        int p;
        float s;
        Raw8<T> row;
    };
    TL t;
    const auto start = [&](int n) {
        const int id = of_xcd(n, total);
        const int4 tile = reinterpret_cast<const int4 *>(a.plan.tiles)[1 + id / across];
        const int e = __builtin_amdgcn_readfirstlane(tile.x);
        const Job j{__builtin_amdgcn_readfirstlane(tile.y), __builtin_amdgcn_readfirstlane(tile.z), id % across * TL::BJ};
        Rows x = a.x, w = a.w;
        if (x.list)
            x.list += j.first;
        else
            x.base += j.first * x.stride;
        x.count = j.rows;
        w.base += e * a.expert;
        t.start(x, w, 0, j.j0, a.inner, lds);
        return j;
    };
    int n = blockIdx.x;
    if (n < total) job = start(n);
    clear_unlisted<TL::kWaves>(a);  // while the first tile's loads are on their way
    if (n >= total) return;
    for (bool landed = false;; landed = true) {
        t.sums(a.inner, job.rows, a.cols - job.j0, landed, lds);
        n += gridDim.x;
        if (n < total) next = start(n);
        t.template each<false>(
            lds,
            [&](int i, int j) {
                Beside b;
                b.p = i < job.rows ? a.plan.pairs[job.first + i] : -1;
                b.s = a.scale && b.p >= 0 ? a.scale[b.p] : 1.0f;
                if (a.dotted)
                    b.row.load(static_cast<const typename T::type *>(a.dotted) + (b.p < 0 ? 0 : b.p) / a.dot_slots * a.lddot +
                                   job.j0 + j,
                               b.p < 0 ? 0 : a.cols - job.j0 - j);
                return b;
            },
            [&](int i, int j, const float (&sums)[8], const Beside &b) {
                const int p = b.p, there = a.cols - job.j0 - j;
                if (a.dotted) {
                    float u[8], d = 0.0f;
                    b.row.widen(u);
#pragma unroll
                    for (int k = 0; k < 8; ++k) d = fmaf(k < there ? sums[k] : 0.0f, u[k], d);
#pragma unroll
                    for (int by = 1; by < TL::kLanes; by *= 2) d += __shfl_xor(d, by);
                    if (j % TL::kCols == 0 && p >= 0 && there > 0)
                        a.dots[static_cast<int64_t>(p) * a.ndots + (job.j0 + j) / TL::kCols] = d;
                }
                if (p < 0 || there <= 0) return;
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[k] = sums[k] * b.s;
                    if (a.relu) v[k] = v[k] < 0.0f ? 0.0f : v[k];  // a NaN stays
                }
                store8_as(a.out, p * a.ldo + job.j0 + j, v, there, a.otype);
            },
            [](int, int, const float (&)[8]) {});
        if (n >= total) return;
        job = next;
    }
}

// The part of a product's arguments that the call's lists make.
inline RowsArgs rows_of(const ExpertArgs &a, Unlisted unlisted) {
    RowsArgs r{};
    r.plan = a.plan;
    r.unlisted = unlisted;
    r.ids = a.ids;
    r.P = static_cast<int>(a.pairs());
    r.E = a.E;
    return r;
}

// Whether a side's rows can go into LDS by direct loads.
inline bool direct_rows(const void *p, int64_t ld, int width, int size) {
    return size == 2 && reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0 && width % 8 == 0 && ld < int64_t{1} << 31;
}

template <class TL>
hipError_t launch_rows(const RowsArgs &a, int64_t pairs, int E, hipStream_t s) {
    if (hipError_t e = allow_lds<expert_rows_kernel<TL>>(TL::kLds); e != hipSuccess) return e;
    const int64_t tiles = pairs / TL::BI + (pairs < E ? pairs : E);  // as many as there can be
    const int64_t all = tiles * ((a.cols + TL::BJ - 1) / TL::BJ), grid = all < kResident<TL> ? all : kResident<TL>;
    hipLaunchKernelGGL(expert_rows_kernel<TL>, dim3(static_cast<unsigned>(grid)), dim3(TL::kThreads), TL::kLds, s, a);
    return hipGetLastError();
}

template <class T, bool DIRECT, Side WS>
hipError_t launch_rows_of(const RowsArgs &a, int64_t pairs, int E, int rows, hipStream_t s) {
    if constexpr (DIRECT)
        if (rows == 256) return launch_rows<Tile<T, true, kAlong, WS, 256, 256, 2, 4>>(a, pairs, E, s);
    if constexpr (!std::is_same_v<T, F32>)
        if (rows == 32) return launch_rows<Tile<T, DIRECT, kAlong, WS, 32, 128, 1, 4>>(a, pairs, E, s);
    if (rows == 64) return launch_rows<Tile<T, DIRECT, kAlong, WS, 64, 64, 2, 2, 0, kInner64<DIRECT>>>(a, pairs, E, s);
    return launch_rows<Tile<T, DIRECT, kAlong, WS, 128, 128, 2, kWavesOf128<T>>>(a, pairs, E, s);
}
template <Side WS>
hipError_t launch_rows_by(const RowsArgs &a, int type, bool direct, int64_t pairs, int E, hipStream_t s) {
    const int rows = expert_tile_rows(pairs, E, a.cols, type, direct);
    if (type == ISC_F32) return launch_rows_of<F32, false, WS>(a, pairs, E, rows, s);
    if (type == ISC_BF16)
        return direct ? launch_rows_of<BF16, true, WS>(a, pairs, E, rows, s)
                      : launch_rows_of<BF16, false, WS>(a, pairs, E, rows, s);
    return direct ? launch_rows_of<F16, true, WS>(a, pairs, E, rows, s)
                  : launch_rows_of<F16, false, WS>(a, pairs, E, rows, s);
}

}  // namespace tp
}  // namespace isc
