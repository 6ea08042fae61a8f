// Products of tokens with the matrices of the experts that a router gave them,
// on weights in 16 or 32 bits (isc_expert_linear), and the launches that they
// share with their gradients (expert_grad.hip).
//
// y[p] = w[e] x[p] for every pair p = (token, slot) of expert e: a matrix product
// for each expert, whose rows are as many as the router gave it.  The first
// launch cuts each expert's pairs into tiles of rows and lists them, the second
// takes a workgroup for every tile of rows by a tile of outputs (tile_product.hpp).
// A sum over a token's slots is a third launch over the pairs' fp32 results, in
// the slots' order: added up by atomics its order would change from run to run.
#include "expert.hpp"

namespace isc {
namespace {

constexpr int kPlanThreads = 256;

// The place of the expert with `rank` others before it, of more pairs, in an order whose eighths,
// one for each XCD, have about as many pairs: dealt to the XCDs there and back, so that each
// has its largest first.  A weight gradient's tiles take as long as their expert has pairs,
// and where an expert's stay together the XCD's L2 serves them (gradients of 64 matrices of
// 1408 x 2048, 512 pairs on average: 316 us, 342 in the experts' own order).
__device__ __forceinline__ int expert_by_size(int rank, int E) {
    const int turn = rank >> 3, xcd = turn & 1 ? 7 - (rank & 7) : rank & 7;
    const int whole = E >> 3, rest = E & 7;  // the last turn has `rest` experts
    const int before = whole & 1 ? (xcd > 8 - rest ? xcd - (8 - rest) : 0) : (xcd < rest ? xcd : rest);
    return xcd * whole + before + turn;
}

// Workgroup 0 lists the tiles, with by_size the last one the experts' order; the others make
// the lists by place.  A place holds a pair if it is one of those of the expert that ids
// gives the pair: whatever `order` says, a row is its own expert's or 0.
__global__ __launch_bounds__(kPlanThreads) void expert_plan_kernel(const ExpertArgs a, int rows, bool by_size) {
    const int tid = threadIdx.x;
    const int P = a.T * a.slots;
    if (by_size && blockIdx.x == gridDim.x - 1) {
        __shared__ __attribute__((aligned(16))) int32_t counts[1024];
        const auto count = [&](int e) {
            const int lo = a.offsets[e], hi = a.offsets[e + 1];
            const int from = lo < 0 ? 0 : lo > P ? P : lo, end = hi > P ? P : hi;
            return end > from ? end - from : 0;
        };
        for (int e = tid; e < (a.E + 3) / 4 * 4; e += kPlanThreads) counts[e] = e < a.E ? count(e) : -1;
        __syncthreads();
        for (int e = tid; e < a.E; e += kPlanThreads) {
            const int own = counts[e];
            int rank = 0;
#pragma unroll 4
            for (int q = 0; q < a.E; q += 4) {
                const int4 other = *reinterpret_cast<const int4 *>(counts + q);
                rank += other.x > own || (other.x == own && q < e);
                rank += other.y > own || (other.y == own && q + 1 < e);
                rank += other.z > own || (other.z == own && q + 2 < e);
                rank += other.w > own || (other.w == own && q + 3 < e);
            }
            a.plan.by_size[expert_by_size(rank, a.E)] = e;
        }
        return;
    }
    if (blockIdx.x == 0) {
        __shared__ int32_t sums[kPlanThreads];
        constexpr int kEach = 4;  // experts of a thread: at most 1024 in all
        int32_t from[kEach], count[kEach], mine = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int e = kEach * tid + i;
            from[i] = count[i] = 0;
            if (e < a.E) {
                const int lo = a.offsets[e], hi = a.offsets[e + 1];
                from[i] = lo < 0 ? 0 : lo > P ? P : lo;
                const int end = hi > P ? P : hi;
                count[i] = end > from[i] ? end - from[i] : 0;
            }
            mine += (count[i] + rows - 1) / rows;
        }
        sums[tid] = mine;
        __syncthreads();
        for (int d = 1; d < kPlanThreads; d *= 2) {
            const int32_t other = tid >= d ? sums[tid - d] : 0;
            __syncthreads();
            sums[tid] += other;
            __syncthreads();
        }
        // lists that overlap could ask for more tiles than a route can have
        const int most = P / rows + (P < a.E ? P : a.E);
        int at = sums[tid] - mine;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            for (int r = 0; r < count[i] && at < most; r += rows, ++at)
                reinterpret_cast<int4 *>(a.plan.tiles)[1 + at] =
                    make_int4(kEach * tid + i, from[i] + r, count[i] - r < rows ? count[i] - r : rows, 0);
        if (tid == kPlanThreads - 1) a.plan.tiles[0] = sums[tid] < most ? sums[tid] : most;
        return;
    }
    const int i = (blockIdx.x - 1) * kPlanThreads + tid;
    if (i >= P) return;
    const int p = a.order[i];
    bool there = static_cast<unsigned>(p) < static_cast<unsigned>(P);
    if (there) {
        const int e = a.ids[p];
        there = static_cast<unsigned>(e) < static_cast<unsigned>(a.E) && i >= a.offsets[e] && i < a.offsets[e + 1];
    }
    a.plan.pairs[i] = there ? p : -1;
    a.plan.tokens[i] = there ? p / a.slots : -1;
    if (there) a.plan.places[p] = i;
}

// Four columns of a token a thread; eight slots' loads in flight.
template <class T>
__global__ __launch_bounds__(256) void expert_sum_kernel(const ExpertArgs a, const float *part, int cols, int64_t ld,
                                                         const float *weights, typename T::type *out, int64_t ldo) {
    const int quads = (cols + 3) / 4;
    const int64_t all = static_cast<int64_t>(a.T) * quads, hop = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all; i += hop) {
        const int64_t t = i / quads;
        const int c = static_cast<int>(i - t * quads) * 4;
        float4 sum = make_float4(0, 0, 0, 0);
        for (int j0 = 0; j0 < a.slots; j0 += 8) {
            float4 v[8];
            float w[8];
            bool there[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t p = t * a.slots + (j0 + j < a.slots ? j0 + j : j0);
                v[j] = *reinterpret_cast<const float4 *>(part + p * ld + c);
                there[j] = j0 + j < a.slots && static_cast<unsigned>(a.ids[p]) < static_cast<unsigned>(a.E);
                w[j] = weights ? weights[p] : 1.0f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (!there[j]) continue;  // a row that nothing wrote, a weight that may be anything
                sum.x = fmaf(w[j], v[j].x, sum.x);
                sum.y = fmaf(w[j], v[j].y, sum.y);
                sum.z = fmaf(w[j], v[j].z, sum.z);
                sum.w = fmaf(w[j], v[j].w, sum.w);
            }
        }
        typename T::type *to = out + t * ldo + c;
        store<T>(to, sum.x);
        if (c + 1 < cols) store<T>(to + 1, sum.y);
        if (c + 2 < cols) store<T>(to + 2, sum.z);
        if (c + 3 < cols) store<T>(to + 3, sum.w);
    }
}

}  // namespace

// By the rows that an expert has on average, of experts that can have any, and the tiles that
// this makes.  Tiles of 256 x 256 need all of a compute unit's LDS, and direct loads.
int expert_tile_rows(int64_t pairs, int E, int cols, int type, bool direct) {
    const int64_t met = pairs < E ? pairs > 0 ? pairs : 1 : E, of_one = pairs / met;
    if (of_one <= 32 && type != ISC_F32) return 32;
    const auto tiles = [&](int side) { return met * ((of_one + side - 1) / side) * ((cols + side - 1) / side); };
    return tp::tile_side(direct && of_one >= 128 ? tiles(256) : 0, tiles(128), type == ISC_F32);
}

namespace {

// Tiles of rows that there can be, whichever kernel runs.
int64_t most_tiles(int64_t pairs, int E) { return pairs / 32 + (pairs < E ? pairs : E); }

}  // namespace

bool expert_launches_fit(int64_t pairs, int E, int N, int K, int type) {
    const int64_t across = ((N > K ? N : K) + 63) / 64;
    return most_tiles(pairs, E) * across < int64_t{1} << 31 &&
           ((N + 63) / 64) * static_cast<int64_t>((K + 63) / 64) * E < int64_t{1} << 31;
}

size_t expert_plan_bytes(int64_t pairs, int E, int type) {
    return static_cast<size_t>((16 * (1 + most_tiles(pairs, E)) + 255) / 256 * 256 + (12 * pairs + 255) / 256 * 256 +
                               (4 * E + 255) / 256 * 256);
}

ExpertPlan expert_plan_at(void *ws, int64_t pairs, int E, int type) {
    ExpertPlan p;
    p.tiles = static_cast<int32_t *>(ws);
    p.pairs = past(p.tiles, (16 * (1 + most_tiles(pairs, E)) + 255) / 256 * 256);
    p.tokens = past(p.pairs, 4 * pairs);
    p.places = past(p.tokens, 4 * pairs);
    p.by_size = past(p.pairs, (12 * pairs + 255) / 256 * 256);
    return p;
}

hipError_t launch_expert_plan(const ExpertArgs &a, int rows, bool by_size, hipStream_t s) {
    const int64_t blocks = 1 + (a.pairs() + kPlanThreads - 1) / kPlanThreads + by_size;
    hipLaunchKernelGGL(expert_plan_kernel, dim3(static_cast<unsigned>(blocks)), dim3(kPlanThreads), 0, s, a, rows,
                       by_size);
    return hipGetLastError();
}

hipError_t launch_expert_sum(const ExpertArgs &a, const float *part, int cols, const float *weights, void *out,
                             int64_t ldo, int type, hipStream_t s) {
    const int64_t all = static_cast<int64_t>(a.T) * ((cols + 3) / 4), blocks = (all + 255) / 256;
    const dim3 grid(static_cast<unsigned>(blocks < 8192 ? blocks : 8192));
    const int64_t ld = expert_ld(cols);
    if (type == ISC_F32)
        hipLaunchKernelGGL(expert_sum_kernel<F32>, grid, dim3(256), 0, s, a, part, cols, ld, weights,
                           static_cast<float *>(out), ldo);
    else if (type == ISC_BF16)
        hipLaunchKernelGGL(expert_sum_kernel<BF16>, grid, dim3(256), 0, s, a, part, cols, ld, weights,
                           static_cast<uint16_t *>(out), ldo);
    else
        hipLaunchKernelGGL(expert_sum_kernel<F16>, grid, dim3(256), 0, s, a, part, cols, ld, weights,
                           static_cast<uint16_t *>(out), ldo);
    return hipGetLastError();
}

hipError_t launch_expert_linear(const ExpertLinearArgs &l, hipStream_t s) {
    const ExpertArgs &a = l.a;
    if (expert_few(a.pairs(), a.E, a.type)) return launch_expert_few(l, s);
    const int size = a.type == ISC_F32 ? 4 : 2;
    const bool direct = tp::direct_rows(a.x, a.ldx, a.K, size) && tp::direct_rows(a.w, a.ldw, a.K, size);
    const int rows = expert_tile_rows(a.pairs(), a.E, a.N, a.type, direct);
    if (hipError_t e = launch_expert_plan(a, rows, false, s); e != hipSuccess) return e;
    tp::RowsArgs r = tp::rows_of(a, l.combine ? tp::kWithExpert : tp::kAll);
    r.x = {static_cast<const char *>(a.x), a.ldx * size, a.shared ? a.plan.tokens : a.plan.pairs, 0, a.K};
    r.w = {static_cast<const char *>(a.w), a.ldw * size, nullptr, a.N, a.K};
    r.expert = a.N * a.ldw * size;
    r.inner = a.K;
    r.cols = a.N;
    r.out = l.combine ? l.part : l.y;
    r.ldo = l.combine ? expert_ld(a.N) : l.ldy;
    r.otype = l.combine ? ISC_F32 : l.ytype;
    r.relu = l.relu;
    if (hipError_t e = tp::launch_rows_by<tp::kAlong>(r, a.type, direct, a.pairs(), a.E, s); e != hipSuccess) return e;
    if (!l.combine) return hipSuccess;
    return launch_expert_sum(a, l.part, a.N, a.weights, l.y, l.ldy, l.ytype, s);
}

}  // namespace isc
