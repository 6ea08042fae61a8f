// isc_expert_linear for few pairs an expert: a decoding step's.
//
// A weight is read once for every 16 pairs of its expert, which has a handful, so the
// time is that of reading the met experts' matrices.  A workgroup takes 16 outputs of an
// expert and up to 16 of its pairs at a time; its wavefronts share the inputs, and every
// lane has its weights of 512 inputs on the way at once: neither LDS nor a first launch
// that lists tiles stands in front of the reads.  The lists are read as they are.
//
// v_mfma_f32_16x16x32 (16 bits): lane l holds 8 r of row l % 16 of either operand.  Which
// 8 is free as long as both agree, so a lane takes 16 consecutive inputs of a step of 64
// in two loads, and the four lanes of a row a whole line.  fp32 takes v_mfma_f32_16x16x4
// on the values as they are: the matrix cores have time.
#include "expert.hpp"

namespace isc {
namespace {

using namespace tp;
using f32x4 = __attribute__((ext_vector_type(4))) float;

constexpr int kWaves = 4;
constexpr int kFewEach = 4, kFewEachWide = 8;  // pairs an expert on average, of 16 and of 32 bits
constexpr int kFewPairs = kFewEachWide * 1024;  // the most that there can be

template <class T>
struct Few {
    static constexpr bool kWide = std::is_same_v<T, F32>;
    static constexpr int kStep = kWide ? 32 : 64;   // inputs of a step
    static constexpr int kAhead = 8;                // steps on their way
    static __device__ __forceinline__ f32x4 product(const Raw8<T> &w, const Raw8<T> &x, f32x4 c) {
        if constexpr (kWide) {
            const uint32_t a[8] = {w.a.x, w.a.y, w.a.z, w.a.w, w.b.x, w.b.y, w.b.z, w.b.w};
            const uint32_t b[8] = {x.a.x, x.a.y, x.a.z, x.a.w, x.b.x, x.b.y, x.b.z, x.b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
            return c;
        } else if constexpr (std::is_same_v<T, BF16>) {
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.a), __builtin_bit_cast(bf16x8, x.a),
                                                           c, 0, 0, 0);
        } else {
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w.a), __builtin_bit_cast(f16x8, x.a), c,
                                                          0, 0, 0);
        }
    }
};

template <class T>
__global__ __launch_bounds__(64 * kWaves) void expert_few_kernel(const ExpertArgs a, void *out, int64_t ldo, int otype,
                                                                 int relu, int zeros) {
    using F = Few<T>;
    using V = typename T::type;
    constexpr int kEach = F::kWide ? 1 : 2;  // loads of a lane and step
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int e = static_cast<int>(blockIdx.y) - 1, n0 = blockIdx.x * 16, P = a.T * a.slots;
    if (e < 0) {  // the rows of pairs that no place of their expert lists become 0
        // to be summed, only those that have an expert, of which there are none as a rule: one workgroup's
        if (!zeros && blockIdx.x) return;
        __shared__ uint32_t kept[kFewPairs / 32];
        const auto has = [&](int p) { return static_cast<unsigned>(a.ids[p]) < static_cast<unsigned>(a.E); };
        for (int i = tid; i < (P + 31) / 32; i += 64 * kWaves) kept[i] = 32 * i + 32 > P ? ~0u << (P & 31) : 0;
        __syncthreads();
        for (int i = tid; i < P; i += 64 * kWaves) {
            if (!zeros && !has(i)) atomicOr(&kept[i >> 5], 1u << (i & 31));
            const int p = a.order[i];
            if (static_cast<unsigned>(p) < static_cast<unsigned>(P) && has(p) && i >= a.offsets[a.ids[p]] &&
                i < a.offsets[a.ids[p] + 1])
                atomicOr(&kept[p >> 5], 1u << (p & 31));
        }
        __syncthreads();
        if (zeros) {
            for (int i = tid; i < P * 16; i += 64 * kWaves) {
                const int p = i >> 4, n = n0 + (i & 15);
                if (!(kept[p >> 5] >> (p & 31) & 1) && n < a.N) store_as(out, p * ldo + n, 0.0f, otype);
            }
            return;
        }
        for (int q = 0; q < (P + 31) / 32; ++q)
            for (uint32_t gone = ~kept[q]; gone; gone &= gone - 1)
                for (int n = tid; n < a.N; n += 64 * kWaves) store_as(out, (32 * q + __ffs(gone) - 1) * ldo + n, 0.0f, otype);
        return;
    }
    const int lo = a.offsets[e], hi = a.offsets[e + 1];
    const int first = lo < 0 ? 0 : lo > P ? P : lo, end = hi > P ? P : hi;
    const int row = n0 + (lane & 15) < a.N ? n0 + (lane & 15) : a.N - 1;
    const V *w = static_cast<const V *>(a.w) + (static_cast<int64_t>(e) * a.N + row) * a.ldw;
    const int mine = lane >> 4;  // of the four parts of a step
    // the inputs in kWaves parts of whole steps
    const int steps = (a.K + F::kStep - 1) / F::kStep;
    const int s0 = steps * wave / kWaves, s1 = steps * (wave + 1) / kWaves;
    __shared__ f32x4 sums[kWaves - 1][64];
    for (int at = first; at < end; at += 16) {
        const int place = at + (lane & 15);
        int p = place < end ? a.order[place] : -1, own = -1;
        if (p >= P) p = -1;
        const V *x = static_cast<const V *>(a.x) + (p < 0 ? 0 : a.shared ? p / a.slots : p) * a.ldx;
        f32x4 sum = {0, 0, 0, 0};
        for (int s = s0; s < s1; s += F::kAhead) {
            Raw8<T> wv[F::kAhead][kEach], xv[F::kAhead][kEach];
#pragma unroll
            for (int q = 0; q < F::kAhead; ++q)
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const int k = (s + q) * F::kStep + (mine * kEach + i) * 8;
                    wv[q][i].load(w + k, s + q < s1 ? a.K - k : 0);
                }
            // asked for in front of x, which is waited for anyway (the 16 tokens' sum 61.2 us, behind x 63.6)
            if (wave == 0 && s == s0 && p >= 0) own = a.ids[p];
#pragma unroll
            for (int q = 0; q < F::kAhead; ++q)
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const int k = (s + q) * F::kStep + (mine * kEach + i) * 8;
                    xv[q][i].load(x + k, s + q < s1 && p >= 0 ? a.K - k : 0);
                }
#pragma unroll
            for (int q = 0; q < F::kAhead; ++q)
#pragma unroll
                for (int i = 0; i < kEach; ++i) sum = F::product(wv[q][i], xv[q][i], sum);
        }
        if (wave == 0 && s0 >= s1 && p >= 0) own = a.ids[p];
        if (at > first) __syncthreads();  // the sums before are read
        if (wave) sums[wave - 1][lane] = sum;
        __syncthreads();
        if (wave == 0 && own == e) {  // a place that holds another's pair counts for nothing
#pragma unroll
            for (int i = 0; i < kWaves - 1; ++i) sum += sums[i][lane];
            const int n = n0 + 4 * mine;  // results 4 * (l / 16) .. + 4 of column l % 16
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v = relu && sum[i] < 0.0f ? 0.0f : sum[i];  // a NaN stays
                if (n + i < a.N) store_as(out, p * ldo + n + i, v, otype);
            }
        }
    }
}

template <class T>
hipError_t launch(const ExpertLinearArgs &l, hipStream_t s) {
    const ExpertArgs &a = l.a;
    hipLaunchKernelGGL(expert_few_kernel<T>,
                       dim3(static_cast<unsigned>((a.N + 15) / 16), static_cast<unsigned>(a.E + 1)),
                       dim3(64 * kWaves), 0, s, a, l.combine ? static_cast<void *>(l.part) : l.y,
                       l.combine ? expert_ld(a.N) : l.ldy, l.combine ? static_cast<int>(ISC_F32) : l.ytype, l.relu, !l.combine);
    return hipGetLastError();
}

}  // namespace

// Up to 4 pairs an expert on average, 8 in fp32 (64 experts of 1408 of 2048, 8 a token, us by
// this kernel and by tiles: 16 tokens 61 and 77, 32 tokens 66 and 83, 64 tokens 85 and 85;
// fp32 at 64 tokens 171 and 249).  The host knows no more of the lists: where a few experts
// have all pairs their weights are read over and over, in less time than an even load takes
// but more than by tiles (512 tokens, 8 of 1024 experts of 512 of 512: even 180 and 107, the
// same 8 experts for all 97 and 17).
bool expert_few(int64_t pairs, int E, int type) { return pairs <= (type == ISC_F32 ? kFewEachWide : kFewEach) * static_cast<int64_t>(E); }

hipError_t launch_expert_few(const ExpertLinearArgs &l, hipStream_t s) {
    const ExpertArgs &a = l.a;
    const hipError_t e = a.type == ISC_F32 ? launch<F32>(l, s) : a.type == ISC_BF16 ? launch<BF16>(l, s) : launch<F16>(l, s);
    if (e != hipSuccess || !l.combine) return e;
    return launch_expert_sum(a, l.part, a.N, a.weights, l.y, l.ldy, l.ytype, s);
}

}  // namespace isc
