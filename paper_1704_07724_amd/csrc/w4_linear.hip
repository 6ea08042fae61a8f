// Products on 4-bit weights for a dense x: y[t][n] = sum_k w[n][k] x[t][k], by
// one matrix or by the experts that tokens were routed to.
//
// The matrix cores take the weights as they are stored.  An 8-bit x meets them
// in one scaled product of 16 outputs x 16 tokens x 128 inputs, both sides'
// group scales applied inside; no weight is unpacked.  A 16- or 32-bit x is cut
// into parts that bfloat16 holds exactly (1 for bfloat16, 2 for fp16, 3 for
// fp32, each the value's next 8 significant bits), each part a column of its
// own: the 16 columns hold 16, 8 or 5 tokens, and the parts' sums are added at
// the end, the small ones first.  The weights are widened to bfloat16 under
// their scale, exactly, two at a time.  All sums are fp32.
//
// A workgroup owns 16 NT outputs and up to MT tiles of columns; its wavefronts
// share the inputs, 512 at a time in turn, and their sums meet in LDS in the
// wavefronts' order, so a result does not depend on timing.
#include "ffn.hpp"

namespace isc {
namespace {

using i32x8 = int __attribute__((ext_vector_type(8)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

constexpr int kMx8 = 0, kBf16 = 1, kF16 = 2, kF32 = 3;  // how x is fed
template <int MODE>
constexpr int kParts = MODE == kF32 ? 3 : MODE == kF16 ? 2 : 1;
template <int MODE>
constexpr int kTokens = 16 / kParts<MODE>;

// Part `part` of v: its leading 8 significant bits, then the next 8, then the
// last (truncated, so no part overflows; bits that are no number stay in the
// first part alone).
template <int MODE>
__device__ __forceinline__ uint32_t part_bits(float v, int part) {
    const uint32_t b = __float_as_uint(v);
    const float hi = __uint_as_float(b & 0xffff0000u);
    if (MODE == kBf16) return b >> 16;
    const bool finite = (b & 0x7f800000u) != 0x7f800000u;
    if (part == 0) return finite ? b >> 16 : (b | (b & 0xffffu ? 0x400000u : 0u)) >> 16;
    float rest = finite ? v - hi : 0.0f;
    if (MODE == kF32 && part == 2) rest -= __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
    return __float_as_uint(rest) >> 16;
}

// Eight inputs of a column from k on, as a bfloat16 operand.
template <int MODE>
__device__ __forceinline__ bf16x8 column8(const void *x, int64_t row, int k, int K, int part, bool there, bool whole) {
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    const int n = there ? K - k : 0;
    if (MODE == kBf16) {
        const uint16_t *p = static_cast<const uint16_t *>(x) + row + k;
        if (n >= 8 && whole) {
            const uint4 v = *reinterpret_cast<const uint4 *>(p);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            for (int i = 0; i < 8; ++i)
                if (i < n) w[i / 2] |= static_cast<uint32_t>(p[i]) << (16 * (i & 1));
        }
    } else if (n > 0) {
        float v[8];
        if (MODE == kF32)
            load8<F32>(v, static_cast<const float *>(x) + row + k, n, whole && n >= 8);
        else
            load8<F16>(v, static_cast<const uint16_t *>(x) + row + k, n, whole && n >= 8);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = part_bits<MODE>(v[2 * i], part) | part_bits<MODE>(v[2 * i + 1], part) << 16;
    }
    return __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
}

// Sixteen bytes of an 8-bit row from k on.
__device__ __forceinline__ uint4 bytes16(const uint8_t *p, int n, bool whole) {
    if (n >= 16 && whole) return *reinterpret_cast<const uint4 *>(p);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    for (int i = 0; i < 16; ++i)
        if (i < n) w[i / 4] |= static_cast<uint32_t>(p[i]) << (8 * (i & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ bf16x2 widen2(uint32_t w, float scale, int which) {
    switch (which) {
    case 0: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    case 1: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    case 2: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    default: return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    }
}

template <int MODE, int NT, int MT>
__global__ void __launch_bounds__(1024) w4_linear_kernel(W4Args a) {
    constexpr int TOK = kTokens<MODE>, P = kParts<MODE>;
    extern __shared__ f32x4 sums[];  // [wavefronts][NT][MT][64]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int g = lane >> 4, col = lane & 15;
    const int64_t tile0 = static_cast<int64_t>(blockIdx.x) * NT;
    const int64_t ntiles = a.w.tiles();
    const int units = static_cast<int>(a.w.units()), steps = static_cast<int>(a.w.steps());
    // the rows of this workgroup: tokens, or an expert's pairs
    const int64_t all = a.slots ? static_cast<int64_t>(a.T) * a.slots : a.T;
    int64_t first = 0, last = a.T;
    const uint8_t *w = a.packed;
    if (a.slots) {
        const int e = blockIdx.y;
        if (e == a.w.E) {  // slots without an expert: their outputs are 0
            for (int64_t p = static_cast<int64_t>(blockIdx.x) * waves + wave; p < all;
                 p += static_cast<int64_t>(gridDim.x) * waves) {
                const int id = a.ids[p];
                if (id >= 0 && id < a.w.E) continue;
                for (int n = lane; n < a.w.N; n += 64) store_as(a.y, p * a.ldy + n, 0.0f, a.ytype);
            }
            return;
        }
        first = a.offsets[e];
        last = a.offsets[e + 1];
        if (first < 0) first = 0;
        if (last > all) last = all;
        w += static_cast<int64_t>(e) * a.w.tile_bytes();
    } else {
        first = static_cast<int64_t>(blockIdx.y) * TOK * MT;
        last = first + TOK * MT < last ? first + TOK * MT : last;
    }
    const uint4 *codes = reinterpret_cast<const uint4 *>(w);
    const uint32_t *scales = reinterpret_cast<const uint32_t *>(w + a.w.tile_codes());

    for (int64_t r0 = first; r0 < last; r0 += TOK * MT) {
        // this lane's column of each tile: a row of x and a part of its values
        int64_t xrow[MT];
        bool there[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int64_t r = r0 + m * TOK + col / P;
            there[m] = r < last && col < TOK * P;
            xrow[m] = 0;
            if (there[m]) {
                const int64_t p = a.slots ? a.order[r] : r;
                there[m] = p >= 0 && p < all;
                if (there[m]) xrow[m] = a.slots ? p / a.slots : p;
            }
        }
        f32x4 acc[NT][MT] = {};
        for (int u = wave; u < units; u += waves) {
            uint32_t sc[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int64_t tile = tile0 + i < ntiles ? tile0 + i : ntiles - 1;
                sc[i] = scales[(tile * units + u) * 64 + lane];
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int step = u * 4 + s;
                if (step >= steps) break;
                uint4 q[NT];
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const int64_t tile = tile0 + i < ntiles ? tile0 + i : ntiles - 1;
                    q[i] = codes[(tile * steps + step) * 64 + lane];
                }
                const int k = step * 128;
                if constexpr (MODE == kMx8) {
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
                        uint32_t xs = 127;
                        if (there[m]) {
                            const uint8_t *x = static_cast<const uint8_t *>(a.x) + xrow[m] * a.ldx;
                            lo = bytes16(x + k + 16 * g, a.w.K - k - 16 * g, a.whole);
                            hi = bytes16(x + k + 64 + 16 * g, a.w.K - k - 64 - 16 * g, a.whole);
                            if (k + 32 * g < a.w.K) xs = a.xs[xrow[m] * a.ldxs + (k >> 5) + g];
                        }
                        const i32x8 b = {static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(lo.z),
                                         static_cast<int>(lo.w), static_cast<int>(hi.x), static_cast<int>(hi.y),
                                         static_cast<int>(hi.z), static_cast<int>(hi.w)};
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            const i32x8 f = {static_cast<int>(q[i].x), static_cast<int>(q[i].y),
                                             static_cast<int>(q[i].z), static_cast<int>(q[i].w), 0, 0, 0, 0};
                            acc[i][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                                f, b, acc[i][m], 4, 0, 0, static_cast<int>(sc[i] >> (8 * s)), 0,
                                static_cast<int>(xs));
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        bf16x8 f[NT];
#pragma unroll
                        for (int i = 0; i < NT; ++i) {
                            const uint32_t word = j == 0 ? q[i].x : j == 1 ? q[i].y : j == 2 ? q[i].z : q[i].w;
                            const float scale = scale_value(sc[i] >> (8 * s) & 255u);
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                const bf16x2 v = widen2(word, scale, c);
                                f[i][2 * c] = v[0];
                                f[i][2 * c + 1] = v[1];
                            }
                        }
#pragma unroll
                        for (int m = 0; m < MT; ++m) {
                            const bf16x8 b = column8<MODE>(a.x, xrow[m] * a.ldx, k + 32 * g + 8 * j, a.w.K, col % P,
                                                           there[m], a.whole);
#pragma unroll
                            for (int i = 0; i < NT; ++i)
                                acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i], b, acc[i][m], 0, 0, 0);
                        }
                    }
                }
            }
        }
        // add the wavefronts' sums up and the parts, and store
        __syncthreads();  // the rows before are stored
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m) sums[((wave * NT + i) * MT + m) * 64 + lane] = acc[i][m];
        __syncthreads();
        const float *flat = reinterpret_cast<const float *>(sums);
        for (int o = threadIdx.x; o < NT * MT * TOK * 16; o += blockDim.x) {
            const int n = o & 15, t = (o >> 4) % TOK, m = (o >> 4) / TOK % MT, i = (o >> 4) / TOK / MT;
            const int64_t r = r0 + m * TOK + t, out = (tile0 + i) * 16 + n;
            if (r >= last || out >= a.w.N) continue;
            float v = 0.0f;
#pragma unroll
            for (int part = P - 1; part >= 0; --part) {
                float u = 0.0f;
                for (int z = 0; z < waves; ++z)
                    u += flat[(((z * NT + i) * MT + m) * 64 + (n >> 2) * 16 + t * P + part) * 4 + (n & 3)];
                v += u;
            }
            if (a.relu && !(v > 0.0f) && v == v) v = 0.0f;
            const int64_t p = a.slots ? a.order[r] : r;
            if (p >= 0 && p < all) store_as(a.y, p * a.ldy + out, v, a.ytype);
        }
    }
}

template <int MODE, int NT, int MT>
hipError_t run(const W4Args &a, hipStream_t s) {
    const int64_t tiles = (a.w.tiles() + NT - 1) / NT;
    const int64_t rows = kTokens<MODE> * MT;
    const unsigned y = static_cast<unsigned>(a.slots ? a.w.E + 1 : (a.T + rows - 1) / rows);
    int waves = 1;
    while (waves < 8 && waves < a.w.units()) waves *= 2;
    const size_t lds = sizeof(float) * 256 * static_cast<size_t>(waves * NT * MT);
    w4_linear_kernel<MODE, NT, MT>
        <<<dim3(static_cast<unsigned>(tiles), y), dim3(static_cast<unsigned>(64 * waves)), lds, s>>>(a);
    return hipGetLastError();
}

template <int MODE>
hipError_t by_tokens(const W4Args &a, hipStream_t s) {
    const int64_t rows = a.slots ? (static_cast<int64_t>(a.T) * a.slots + a.w.E - 1) / a.w.E : a.T;
    if (rows <= kTokens<MODE>) return run<MODE, 1, 1>(a, s);
    if (rows <= 2 * kTokens<MODE>) return run<MODE, 1, 2>(a, s);
    return run<MODE, 1, 4>(a, s);
}

}  // namespace

hipError_t launch_w4_linear(const W4Args &a, hipStream_t s) {
    switch (a.xtype) {
    case ISC_MX8: return by_tokens<kMx8>(a, s);
    case ISC_BF16: return by_tokens<kBf16>(a, s);
    case ISC_F16: return by_tokens<kF16>(a, s);
    default: return by_tokens<kF32>(a, s);
    }
}

}  // namespace isc
