// Routing of tokens to experts, and its gradient.
//
//   s = softmax(l) or 1 / (1 + exp(-l)),  key = s + bias
//   a group's key: the sum of its two largest keys; the best groups stay
//   the k largest keys of those, ties to the lowest index
//   w_j = scale s_j / (sum of the chosen s + 1e-20), or scale s_j
//
// An expert whose logit (or key) is -inf or NaN is never chosen; a token with
// fewer than k experts left gets id -1 and weight 0 in its last slots.
//
// LANES lanes share a token, 64 or (many tokens, at most 256 experts, 16 slots
// and groups) 16, so that a wavefront routes four.  The keys stay in registers
// as unsigned integers in the floats' order, the experts of a lane LANES apart;
// a slot is a maximum and then a minimum of the indices that have it, by
// data-parallel moves.  A token's slots wait for each other, and that bounds all
// but the largest calls: 16 tokens of 256 experts in groups take 9.1 us, 4096
// tokens 14.0, 8192 of 128 experts with their lists 11.6, where moving the 3 MB
// would take one; 16384 of 256 in groups, where the instructions count, 24.9.
//
// The experts' lists.  A token meets an expert at most once, so 64 tokens and
// an expert make one 64-bit word: a pair's place among its expert's pairs is
// the number of bits below its token's, whatever order the bits were set in.
// Workgroups of 16 to 64 tokens leave their counts; a second launch, of 64 tokens
// a workgroup, adds up the counts of the workgroups before, and the experts'
// totals, and places pairs.
#include "ffn.hpp"

#include <atomic>

namespace isc {
namespace {

constexpr int kWaves = 16;    // wavefronts per workgroup
constexpr int kMaxE = 1024;   // experts, and threads of a workgroup

// Reductions over a token's lanes.
template <int LANES>
__device__ __forceinline__ uint32_t max_of(uint32_t v) {
    return LANES == 16 ? row_max(v) : wave_max(v);
}
template <int LANES>
__device__ __forceinline__ uint32_t min_of(uint32_t v) {
    return LANES == 16 ? row_min(v) : wave_min(v);
}
template <int LANES>
__device__ __forceinline__ float sum_of(float v) {
    return LANES == 16 ? row_sum(v) : wave_sum(v);
}

// e^x for x <= 0, down to the smallest fp32 number: e^x = 2^n 2^f with n the nearest
// whole number to x log2 e and |f| <= 1/2, the product with log2 e in two parts, so the
// error stays near one unit in the last place; 2^n goes on last, since the instruction
// has no results below 2^-126.
// (A third of the instructions of the library's: a kernel that routes a few
// tokens waits for its own code to arrive more than for anything else.)
__device__ __forceinline__ float exponential(float x) {
    x = __builtin_amdgcn_fmed3f(x, -104.0f, 0.0f);  // (0 from there down)
    const float n = __builtin_rintf(x * 0x1.715476p+0f);
    const float f = fmaf(x, 0x1.4ae0cp-26f, fmaf(x, 0x1.715476p+0f, -n));
    return __builtin_ldexpf(__builtin_amdgcn_exp2f(f), static_cast<int>(n));
}

// s = 1 / (1 + e^-l) and s (1 - s), both from e^-|l| <= 1: neither comes from a
// difference, and each has a value wherever fp32 has one.
struct Sigmoid {
    float s, slope;
};
__device__ __forceinline__ Sigmoid sigmoid_of(float l) {
    const float e = exponential(-fabsf(l)), r = __builtin_amdgcn_rcpf(1.0f + e);
    return {l < 0.0f ? e * r : r, e * r * r};
}

// A token's scores from its logits, expert i * LANES + lane in place i, written
// over them; -1 for a logit that is not above -inf.  A logit of +inf stands for
// all others' limit: it shares the softmax with its equals.  Returns the softmax's
// largest logit.
template <int C, int LANES>
__device__ __forceinline__ float scores(float (&s)[C], int sigmoid) {
    if (sigmoid) {
#pragma unroll
        for (int i = 0; i < C; ++i) s[i] = s[i] > -__builtin_inff() ? sigmoid_of(s[i]).s : -1.0f;
        return 0.0f;
    }
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < C; ++i)
        if (s[i] > -__builtin_inff()) mx = op_max(mx, order(s[i]));
    mx = max_of<LANES>(mx);
    const float m = mx ? unorder(mx) : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const bool there = s[i] > -__builtin_inff();
        s[i] = there ? (s[i] == m ? 1.0f : exponential(s[i] - m)) : -1.0f;
        sum += there ? s[i] : 0.0f;
    }
    sum = sum_of<LANES>(sum);
    const float inv = sum > 0.0f ? 1.0f / sum : 1.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) s[i] = s[i] < 0.0f ? s[i] : s[i] * inv;
    return m;
}

// A token's logits, -inf past the last expert.
template <int C, int LANES>
__device__ __forceinline__ void load_logits(float (&l)[C], const void *logits, int64_t at, int lane, int E, int type) {
    uint32_t raw[C];
    if (type == ISC_F32) {
        const uint32_t *p = static_cast<const uint32_t *>(logits) + at;
#pragma unroll
        for (int i = 0; i < C; ++i) raw[i] = p[i * LANES + lane < E ? i * LANES + lane : 0];
    } else {
        const uint16_t *p = static_cast<const uint16_t *>(logits) + at;
#pragma unroll
        for (int i = 0; i < C; ++i) raw[i] = p[i * LANES + lane < E ? i * LANES + lane : 0];
    }
#pragma unroll
    for (int i = 0; i < C; ++i) {
        l[i] = type == ISC_F16 ? F16::widen(raw[i]) : __uint_as_float(type == ISC_BF16 ? raw[i] << 16 : raw[i]);
        if (i * LANES + lane >= E) l[i] = -__builtin_inff();
    }
}

__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Token t by LANES lanes, all of the wavefront's tokens together (t past the
// last one routes the last again and stores nothing); `row` is E words of LDS
// of the token's own, used with groups only.  Lane j < k of the token returns
// slot j's expert, or -1.
template <int C, int LANES>
__device__ __forceinline__ int route_token(const RouteArgs &a, int64_t t, uint32_t *row) {
    const int lane = threadIdx.x & (LANES - 1), first = threadIdx.x & 63 & ~(LANES - 1);
    const bool there = t < a.T;
    const int64_t at = there ? t : a.T - 1;
    float s[C];
    uint32_t key[C];  // 0: not to be chosen
    // with sixteen experts a lane the logits' addresses are made again for each token:
    // kept from one to the next they do not fit the registers
    int from = lane;
    if constexpr (LANES * C == kMaxE) asm volatile("" : "+v"(from));
    load_logits<C, LANES>(s, a.logits, at * a.ld, from, a.E, a.type);
    // without a bias the logits rank as their scores do, and also where fp32's scores
    // are equal: near a sigmoid of 1, and below 2^-149
    if (!a.bias)
#pragma unroll
        for (int i = 0; i < C; ++i) key[i] = s[i] > -__builtin_inff() ? order(s[i] + 0.0f) : 0u;
    const float m = scores<C, LANES>(s, a.sigmoid);
    if (a.bias) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int e = i * LANES + lane;
            const float v = e < a.E ? s[i] + a.bias[e] : s[i];
            key[i] = s[i] >= 0.0f && v > -__builtin_inff() ? order(v + 0.0f) : 0u;
        }
    } else if (m == __builtin_inff()) {  // beside a logit of +inf the others' scores are 0, all alike
#pragma unroll
        for (int i = 0; i < C; ++i) key[i] = s[i] >= 0.0f ? order(s[i]) : 0u;
    }
    if (a.groups > 1) {
        const int size = a.E / a.groups;
        // e / size as a product: exact, as e times the factor's excess stays below 2^20 / size
        const uint32_t factor = ((1u << 20) + static_cast<uint32_t>(size) - 1u) / static_cast<uint32_t>(size);
#pragma unroll
        for (int i = 0; i < C; ++i)
            if (i * LANES + lane < a.E) row[i * LANES + lane] = key[i] && !a.bias ? order(s[i]) : key[i];
        wave_fence();
        // a group's two largest keys, by the lanes that share it: a power of two
        const int share = LANES >> (32 - __builtin_clz(a.groups - 1));
        const int of = lane / share;  // the lane's group
        uint32_t best = 0, second = 0;
        if (of < a.groups)
#pragma unroll 4
            for (int i = lane % share; i < size; i += share) {
                const uint32_t v = row[of * size + i];
                second = op_max(second, op_min(best, v));
                best = op_max(best, v);
            }
        for (int d = 1; d < share; d <<= 1) {
            const uint32_t b = __shfl_xor(best, d), c = __shfl_xor(second, d);
            second = op_max(op_min(best, b), op_max(second, c));
            best = op_max(best, b);
        }
        wave_fence();
        // 0: none of its experts can be chosen
        if (lane % share == 0 && of < a.groups)
            row[of] = best ? order(unorder(best) + (second ? unorder(second) : 0.0f) + 0.0f) : 0u;
        wave_fence();
        const uint32_t g = lane < a.groups ? row[lane] : 0u;  // lane g's group
        int before = 0;  // groups ranked before the lane's
        for (int j = 0; j < a.groups; ++j) {
            const uint32_t v = row[j];
            before += v > g || (v == g && j < lane);
        }
        const unsigned long long kept = __ballot(lane < a.groups && g && before < a.keep) >> first;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int e = i * LANES + lane;
            if (e < a.E && !(kept >> (static_cast<uint32_t>(e) * factor >> 20) & 1)) key[i] = 0u;
        }
    }
    int id = -1;
    for (int j = 0; j < a.k; ++j) {
        uint32_t best = key[0];
        int e = lane;
#pragma unroll
        for (int i = 1; i < C; ++i)
            if (key[i] > best) best = key[i], e = i * LANES + lane;
        const uint32_t top = max_of<LANES>(best);
        // equal keys in several lanes: the lowest index
        if constexpr (LANES == 64) {
            const unsigned long long tied = __ballot(best == top);
            if (tied & (tied - 1))
                e = static_cast<int>(wave_min(best == top ? static_cast<uint32_t>(e) : 0xffffffffu));
            else
                e = __builtin_amdgcn_readlane(e, __builtin_ctzll(tied));
        } else {
            e = static_cast<int>(row_min(best == top ? static_cast<uint32_t>(e) : 0xffffffffu));
        }
        if (top == 0u) e = -1;  // none is left
#pragma unroll
        for (int i = 0; i < C; ++i)
            if (e == i * LANES + lane) key[i] = 0u;
        if (lane == j) id = e;
    }
    float w = 0.0f;  // the slot's score, from the lane that holds it
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const float v = __shfl(s[i], first + (id & (LANES - 1)));
        if (id >= 0 && id / LANES == i) w = v;
    }
    if (a.renorm) w = w / (sum_of<LANES>(w) + 1e-20f);
    if (!there) return -1;
    if (lane < a.k) {
        a.ids[t * a.k + lane] = id;
        a.weights[t * a.k + lane] = w * a.scale;
    }
    return id;
}

// Exclusive sum of one value per thread over the workgroup of kMaxE threads.
__device__ __forceinline__ int block_scan(int v, int *sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int in = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(in, d);
        if (lane >= d) in += u;
    }
    if (lane == 63) sums[wave] = in;
    __syncthreads();
    int before = 0;
    for (int i = 0; i < wave; ++i) before += sums[i];
    return before + in - v;
}

// Tokens of a workgroup.  One launch does for 16 tokens, and for 64 of at most
// 128 experts (40 of 128: 8.1 us against 8.5 with two).  Else 16 tokens, then 32,
// while that makes no more workgroups than compute units, or 64 (8 of 400 experts
// at 4096 tokens 16.8, 21.5, 31.7 us, in that order; at 8192 26.6, 23.8, 33.2; at
// 16384 46.7, 41.6, 36.9).
int tokens_of(int T, int E) {
    return T > 8192 || (T <= 64 && E <= 128) ? 64 : T > 4096 ? 32 : 16;
}

int blocks_of(int T, int E) {
    const int tokens = tokens_of(T, E);
    return T > tokens ? (T + tokens - 1) / tokens : 1;
}

// A workgroup's counts: whole words of four.
__host__ __device__ constexpr int count_stride(int E) { return (E + 3) & ~3; }

// Routes TOKENS tokens a workgroup.  ONE: there is one workgroup, which also
// writes the lists; else it leaves its counts for place_kernel.
template <int C, int LANES, int THREADS, int TOKENS, bool ONE>
__global__ void __launch_bounds__(THREADS) route_kernel(RouteArgs a) {
    constexpr int kAtOnce = THREADS / LANES, kTurns = TOKENS / kAtOnce;  // tokens at once, and how often
    extern __shared__ uint32_t rows[];  // kAtOnce rows of E words, with groups
    __shared__ unsigned long long bits[kMaxE];
    const int lane = threadIdx.x & (LANES - 1);
    const int own = LANES == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x / LANES;
    const bool lists = a.order != nullptr;
    if (lists) {
        for (int e = threadIdx.x; e < a.E; e += THREADS) bits[e] = 0ull;
        __syncthreads();
    }
    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * TOKENS;
#pragma unroll 1
    for (int i = 0; i < kTurns; ++i) {
        const int t = i * kAtOnce + own;
        // (a whole wavefront without tokens has nothing to do)
        if (t0 + i * kAtOnce + static_cast<int>(threadIdx.x >> 6) * (64 / LANES) >= a.T) break;
        const int id = route_token<C, LANES>(a, t0 + t, rows + own * a.E);
        if (lists && lane < a.k && id >= 0) atomicOr(&bits[id], 1ull << t);
    }
    if (!lists) return;
    __syncthreads();
    if constexpr (!ONE) {
        const int stride = count_stride(a.E);
        for (int e = threadIdx.x; e < stride; e += THREADS)
            a.counts[static_cast<int64_t>(blockIdx.x) * stride + e] = static_cast<uint16_t>(e < a.E ? __popcll(bits[e]) : 0);
    } else {
        static_assert(THREADS == kMaxE);
        __shared__ int base[kMaxE], sums[kWaves], total;
        const int e = threadIdx.x;
        const int count = e < a.E ? __popcll(bits[e]) : 0;
        base[e] = block_scan(count, sums);
        if (e < a.E) a.offsets[e] = base[e];
        if (e == kMaxE - 1) {
            total = base[e] + count;
            a.offsets[a.E] = total;
        }
        __syncthreads();
        const int pairs = a.T * a.k;
        for (int p = threadIdx.x; p < pairs; p += kMaxE) {  // written by this workgroup, before the barriers
            const int id = a.ids[p], t = p / a.k;
            if (id >= 0) a.order[base[id] + __popcll(bits[id] & ((1ull << t) - 1))] = p;
        }
        for (int p = total + static_cast<int>(threadIdx.x); p < a.T * a.k; p += kMaxE) a.order[p] = -1;
    }
}

// The lists of several workgroups' tokens, `tokens` each.
__global__ void __launch_bounds__(kMaxE) place_kernel(RouteArgs a, int tokens) {
    __shared__ unsigned long long bits[kMaxE];
    __shared__ int base[kMaxE], all[kMaxE], sums[kWaves], total;
    const int nb = (a.T + tokens - 1) / tokens, own = 64 / tokens;  // workgroups that routed, and those of this one's tokens
    const int b = blockIdx.x;
    bits[threadIdx.x] = 0ull;
    base[threadIdx.x] = all[threadIdx.x] = 0;
    __syncthreads();
    const int64_t p0 = static_cast<int64_t>(b) * 64 * a.k;
    const int64_t left = static_cast<int64_t>(a.T) * a.k - p0;
    const int pairs = static_cast<int>(left < 64 * a.k ? left : 64 * a.k);
    for (int p = threadIdx.x; p < pairs; p += kMaxE) {
        const int id = a.ids[p0 + p];
        if (id >= 0) atomicOr(&bits[id], 1ull << (p / a.k));
    }
    // threads share the counts: each four experts of every `step`-th workgroup
    // (integer sums: any order gives the same)
    const int quads = count_stride(a.E) / 4, step = kMaxE / quads;
    if (static_cast<int>(threadIdx.x) < step * quads) {
        const int q = threadIdx.x % quads;
        const uint2 *counts = reinterpret_cast<const uint2 *>(a.counts) + q;
        int before[4] = {}, n[4] = {};
        for (int i = threadIdx.x / quads; i < nb; i += 8 * step) {
            uint2 c[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) c[j] = counts[static_cast<int64_t>(i + j * step < nb ? i + j * step : i) * quads];
            uint2 u = {}, v = {};  // two counts a word: eight of at most 64 stay below 2^16
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (i + j * step < nb) u.x += c[j].x, u.y += c[j].y;
                if (i + j * step < b * own) v.x += c[j].x, v.y += c[j].y;
            }
            n[0] += u.x & 0xffff, n[1] += u.x >> 16, n[2] += u.y & 0xffff, n[3] += u.y >> 16;
            before[0] += v.x & 0xffff, before[1] += v.x >> 16, before[2] += v.y & 0xffff, before[3] += v.y >> 16;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            atomicAdd(&all[4 * q + j], n[j]);
            atomicAdd(&base[4 * q + j], before[j]);
        }
    }
    __syncthreads();
    const int e = threadIdx.x;
    const int n = all[e];
    const int start = block_scan(n, sums);
    base[e] += start;
    if (b == 0 && e < a.E) a.offsets[e] = start;
    if (e == kMaxE - 1) {
        total = start + n;
        if (b == 0) a.offsets[a.E] = total;
    }
    __syncthreads();
    for (int p = threadIdx.x; p < pairs; p += kMaxE) {
        const int id = a.ids[p0 + p];
        if (id >= 0)
            a.order[base[id] + __popcll(bits[id] & ((1ull << (p / a.k)) - 1))] = static_cast<int>(p0) + p;
    }
    // the unused tail, spread over the workgroups
    for (int64_t p = total + static_cast<int64_t>(b) * kMaxE + threadIdx.x; p < static_cast<int64_t>(a.T) * a.k;
         p += static_cast<int64_t>(gridDim.x) * kMaxE)
        a.order[p] = -1;
}

// dlogits of four tokens a workgroup, one wavefront each.
template <int C>
__global__ void __launch_bounds__(256) route_bwd_kernel(RouteBwdArgs a) {
    extern __shared__ float grad[];  // four rows of E: the chosen scores' gradients
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * 4 + wave;
    if (t >= a.T) return;
    float *row = grad + wave * a.E;
    float s[C];
    load_logits<C, 64>(s, a.logits, t * a.ld, lane, a.E, a.type);
#pragma unroll
    for (int i = 0; i < C; ++i)
        if (i * 64 + lane < a.E) row[i * 64 + lane] = 0.0f;
    int id = lane < a.k ? a.ids[t * a.k + lane] : -1;
    if (id >= a.E) id = -1;
    float dw = id >= 0 ? a.dweights[t * a.k + lane] * a.scale : 0.0f;
    float slope[C];  // the sigmoid's
    if (a.sigmoid) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const Sigmoid g = sigmoid_of(s[i]);
            const bool there = s[i] > -__builtin_inff();
            s[i] = there ? g.s : 0.0f;
            slope[i] = there ? g.slope : 0.0f;
        }
    } else {
        scores<C, 64>(s, 0);
#pragma unroll
        for (int i = 0; i < C; ++i) s[i] = fmaxf(s[i], 0.0f);
    }
    float chosen = 0.0f;  // slot `lane`'s score, from the lane that holds it
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const float v = __shfl(s[i], id & 63);
        if (id >= 0 && id >> 6 == i) chosen = v;
    }
    // A slot with more than half of a sum meets mostly its own gradient in it, and the
    // difference of the two would be lost in their rounding.  But the gradients add up to
    // a known sum: such a slot's is that less the others'.
    float ds = dw, dot = 0.0f;
    unsigned long long most = 0ull;  // the lane of that slot, for the softmax's own sum
    if (a.renorm) {
        const float total = wave_sum(chosen) + 1e-20f;
        const float mean = wave_sum(dw * chosen) / total;
        ds = (dw - mean) / total;
        dot = mean * (1e-20f / total);  // the sum of ds s
        const bool own = chosen > 0.5f * total;
        if (__ballot(own)) {
            const float others = wave_sum(own ? 0.0f : ds * chosen);
            if (own) ds = (dot - others) / chosen;
        }
    } else if (!a.sigmoid) {
        dot = wave_sum(ds * chosen);
        most = __ballot(chosen > 0.5f);
    }
    if (id < 0) ds = 0.0f;
    __builtin_amdgcn_wave_barrier();
    if (id >= 0) row[id] = ds;  // an expert of its own for every lane
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    float v[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const float d = i * 64 + lane < a.E ? row[i * 64 + lane] : 0.0f;
        v[i] = a.sigmoid ? d * slope[i] : s[i] * (d - dot);
    }
    if (most) {
        const int own = __builtin_amdgcn_readlane(id, __builtin_ctzll(most));
        float others = 0.0f;
#pragma unroll
        for (int i = 0; i < C; ++i) others += i * 64 + lane == own ? 0.0f : v[i];
        others = wave_sum(others);
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] = i * 64 + lane == own ? -others : v[i];
    }
#pragma unroll
    for (int i = 0; i < C; ++i)
        if (i * 64 + lane < a.E) store_as(a.dlogits, t * a.ldd + i * 64 + lane, v[i], a.type);
}

// Grants a kernel the most dynamic LDS a call can ask for, once.
template <typename Kern>
hipError_t grant_lds(Kern kern, std::atomic<bool> &granted, size_t asked) {
    if (asked <= 32 * 1024 || granted.load(std::memory_order_acquire)) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kern),
                                             hipFuncAttributeMaxDynamicSharedMemorySize,
                                             static_cast<int>(sizeof(uint32_t)) * kWaves * kMaxE);
    if (e == hipSuccess) granted.store(true, std::memory_order_release);
    return e;
}

template <int C, int LANES, int THREADS, int TOKENS, bool ONE>
hipError_t route_with(const RouteArgs &a, int blocks, hipStream_t s) {
    static std::atomic<bool> granted{false};
    const size_t lds = a.groups > 1 ? sizeof(uint32_t) * (THREADS / LANES) * static_cast<size_t>(a.E) : 0;
    if (const hipError_t e = grant_lds(route_kernel<C, LANES, THREADS, TOKENS, ONE>, granted, lds); e != hipSuccess) return e;
    route_kernel<C, LANES, THREADS, TOKENS, ONE><<<dim3(static_cast<unsigned>(blocks)), dim3(THREADS), lds, s>>>(a);
    return hipGetLastError();
}

template <int C, int LANES, int THREADS, int TOKENS>
hipError_t route_of(const RouteArgs &a, hipStream_t s) {
    const int nb = blocks_of(a.T, a.E);
    if (nb == 1) return route_with<C, LANES, kMaxE, 64, true>(a, 1, s);
    const hipError_t e = route_with<C, LANES, THREADS, TOKENS, false>(a, nb, s);
    if (e != hipSuccess || !a.order) return e;
    place_kernel<<<dim3(static_cast<unsigned>((a.T + 63) / 64)), dim3(kMaxE), 0, s>>>(a, TOKENS);
    return hipGetLastError();
}
template <int C>
hipError_t one_at_a_time(const RouteArgs &a, hipStream_t s) {
    const int tokens = tokens_of(a.T, a.E);
    return tokens == 16   ? route_of<C, 64, kMaxE, 16>(a, s)
           : tokens == 32 ? route_of<C, 64, kMaxE, 32>(a, s)
                          : route_of<C, 64, kMaxE, 64>(a, s);
}

template <int C>
hipError_t four_at_a_time(const RouteArgs &a, hipStream_t s) {
    return tokens_of(a.T, a.E) == 32 ? route_of<C, 16, 512, 32>(a, s) : route_of<C, 16, kMaxE, 64>(a, s);
}

template <int C>
hipError_t route_bwd_of(const RouteBwdArgs &a, hipStream_t s) {
    const size_t lds = sizeof(float) * 4 * static_cast<size_t>(a.E);
    constexpr int64_t most = kLaunchThreads / 256 * 4;  // tokens of a launch: 2^26 - 4
    const int64_t size = a.type == ISC_F32 ? 4 : 2;
    for (int64_t t0 = 0; t0 < a.T; t0 += most) {
        RouteBwdArgs part = a;
        part.T = static_cast<int>(a.T - t0 < most ? a.T - t0 : most);
        part.dweights = past(a.dweights, t0 * a.k * 4), part.ids = past(a.ids, t0 * a.k * 4);
        part.logits = past(a.logits, t0 * a.ld * size), part.dlogits = past(a.dlogits, t0 * a.ldd * size);
        route_bwd_kernel<C><<<dim3(static_cast<unsigned>((int64_t{part.T} + 3) / 4)), dim3(256), lds, s>>>(part);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t route_count_bytes(int T, int E) {
    const int blocks = blocks_of(T, E);
    return blocks > 1 ? sizeof(uint16_t) * static_cast<size_t>(blocks) * static_cast<size_t>(count_stride(E)) : 0;
}

hipError_t launch_route(const RouteArgs &a, hipStream_t s) {
    // Four tokens a wavefront take fewer instructions a token, one a wavefront
    // fewer in a row: the one where there are tokens enough for every wavefront,
    // the other below (8 of 256 experts in groups at 4096 tokens 18.1 and 14.2 us,
    // at 8192 19.5 and 20.1), but for a single workgroup (40 tokens of 128
    // experts: 8.1 and 9.4 us; up to 16 tokens there is a wavefront for each).
    if (tokens_of(a.T, a.E) > 16 && a.T > kWaves && a.E <= 256 && a.k <= 16 && a.groups <= 16)
        return a.E <= 64 ? four_at_a_time<4>(a, s) : a.E <= 128 ? four_at_a_time<8>(a, s) : four_at_a_time<16>(a, s);
    return a.E <= 64    ? one_at_a_time<1>(a, s)
           : a.E <= 128 ? one_at_a_time<2>(a, s)
           : a.E <= 256 ? one_at_a_time<4>(a, s)
           : a.E <= 512 ? one_at_a_time<8>(a, s)
                        : one_at_a_time<16>(a, s);
}

hipError_t launch_route_bwd(const RouteBwdArgs &a, hipStream_t s) {
    const int c = (a.E + 63) / 64;
    return c <= 1 ? route_bwd_of<1>(a, s)
           : c <= 2 ? route_bwd_of<2>(a, s)
           : c <= 4 ? route_bwd_of<4>(a, s)
           : c <= 8 ? route_bwd_of<8>(a, s)
                    : route_bwd_of<16>(a, s);
}

}  // namespace isc
