// Products on 4-bit weights for a dense x: y[t][n] = sum_k w[n][k] x[t][k], by
// one matrix or by the experts that tokens were routed to.
//
// Both operands become bfloat16 without losing a bit, on the way from memory
// to the matrix cores: a weight has two significant bits and an 8-bit x four,
// each widened under its group's scale, two values an instruction; a 16- or
// 32-bit x is cut into parts of its next 8 significant bits (1 for bfloat16, 2
// for fp16, 3 for fp32).  Each part is a column of its own: the 16 columns of a
// matrix instruction hold 16, 8 or 5 tokens, and the parts' sums are added at
// the end, the small ones first.  Products are then exact and sums are fp32.
// (The scaled 8-bit matrix instruction would take both sides as they are
// stored, but it adds neighbouring products in fewer bits than fp32: 2^-6 next
// to 2^8 is lost.)
//
// A workgroup owns 16 NT outputs and MT tiles of columns; its wavefronts share
// the inputs, 128 at a time in turn, and their sums meet in LDS in the
// wavefronts' order, so a result does not depend on timing.  A wavefront holds
// DEPTH steps' operands in registers, loads in flight behind the matrix work.
#include "ffn.hpp"

#include <type_traits>

namespace isc {
namespace {

using f32x4 = float __attribute__((ext_vector_type(4)));
using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

constexpr int kMx8 = 0, kBf16 = 1, kF16 = 2, kF32 = 3;  // how x is fed
template <int MODE>
constexpr int kParts = MODE == kF32 ? 3 : MODE == kF16 ? 2 : 1;
template <int MODE>
constexpr int kTokens = 16 / kParts<MODE>;
// 16- and 32-bit floats other than bfloat16 go through LDS, cut into parts once.
template <int MODE>
constexpr bool kStaged = MODE >= kF16;
// 32-bit words of a step's inputs that a lane loads: a column's 32 inputs as they
// stand, or for a staged type two neighbouring inputs of every token.
template <int MODE>
constexpr int kWords = MODE == kMx8 ? 8 : MODE == kBf16 ? 16 : MODE == kF16 ? kTokens<kF16> : 2 * kTokens<kF32>;
constexpr int kStageRow = 272;  // bytes of a staged column's 128 inputs; 16 spare spread the columns over the banks
constexpr int kStageTile = 16 * kStageRow;

// One step's operands of a wavefront, as loaded.
template <int MODE, int NT, int MT>
struct Step {
    uint4 q[NT];
    uint32_t sw[NT];
    uint32_t x[MT][kWords<MODE>];
    uint32_t sx[MODE == kMx8 ? MT : 1];
};

// A column's inputs of one step: eight from 32 j + 8 g on for each j, k the
// first.  WHOLE: all of them are there, and aligned.
template <int MODE, bool WHOLE>
__device__ __forceinline__ void load_column(uint32_t (&x)[kWords<MODE>], const uint8_t *row, int k, int K) {
    constexpr int per = kWords<MODE> / 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int at = k + 32 * j;
        if constexpr (WHOLE && MODE == kMx8) {
            const uint2 v = *reinterpret_cast<const uint2 *>(row + at);
            x[j * per] = v.x;
            x[j * per + 1] = v.y;
        } else if constexpr (WHOLE) {
            const uint4 v = *reinterpret_cast<const uint4 *>(row + 2 * at);
            x[j * per] = v.x;
            x[j * per + 1] = v.y;
            x[j * per + 2] = v.z;
            x[j * per + 3] = v.w;
        } else {
#pragma unroll
            for (int i = 0; i < per; ++i) x[j * per + i] = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (at + i >= K) continue;
                if constexpr (MODE == kMx8)
                    x[j * per + i / 4] |= static_cast<uint32_t>(row[at + i]) << (8 * (i & 3));
                else
                    x[j * per + i / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(row)[at + i])
                                          << (16 * (i & 1));
            }
        }
    }
}

// A token's inputs of one step, a staged type's: k and k + 1.
template <int MODE, bool WHOLE>
__device__ __forceinline__ void load_pair(uint32_t *x, const uint8_t *row, int k, int K) {
    if constexpr (MODE == kF32) {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(row) + k;
        if constexpr (WHOLE) {
            const uint2 v = *reinterpret_cast<const uint2 *>(p);
            x[0] = v.x;
            x[1] = v.y;
        } else {
            x[0] = k < K ? p[0] : 0u;
            x[1] = k + 1 < K ? p[1] : 0u;
        }
    } else {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(row) + k;
        if constexpr (WHOLE)
            x[0] = *reinterpret_cast<const uint32_t *>(p);
        else
            x[0] = (k < K ? p[0] : 0u) | (k + 1 < K ? static_cast<uint32_t>(p[1]) : 0u) << 16;
    }
}

__device__ __forceinline__ float scale_word(uint32_t s, int j) {
    // the conversions read the exponent alone: 0 is 2^-127, 255 is NaN
    return __uint_as_float((j == 3 ? s >> 1 : s << (23 - 8 * j)) & 0x7f800000u);
}

// The parts of two values, truncated (so none overflows), as bfloat16 pairs.
// What is no number stays in the first part alone, quiet if it is a NaN.
template <int P>
__device__ __forceinline__ void cut(uint32_t (&w)[P], float a, float b) {
    float v[2] = {a, b};
    uint32_t bits[P][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool number = fabsf(v[i]) < __builtin_inff();
        if (!number) v[i] += v[i];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            bits[p][i] = __float_as_uint(v[i]);
            v[i] = number ? v[i] - __uint_as_float(bits[p][i] & 0xffff0000u) : 0.0f;
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) w[p] = __builtin_amdgcn_perm(bits[p][1], bits[p][0], 0x07060302u);
}

// The bfloat16 operand of eight inputs of a column.
template <int MODE>
__device__ __forceinline__ bf16x8 operand(const uint32_t *x, uint32_t sx, int j) {
    if constexpr (MODE == kBf16) {
        return __builtin_bit_cast(bf16x8, make_uint4(x[0], x[1], x[2], x[3]));
    } else {
        const float s = scale_word(sx, j);
        return __builtin_bit_cast(
            bf16x8, make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[0], s, false)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[0], s, true)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[1], s, false)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[1], s, true))));
    }
}

__device__ __forceinline__ bf16x8 widen8(uint32_t w, float s) {
    const uint4 v = make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)),
                               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3)));
    return __builtin_bit_cast(bf16x8, v);
}

template <int MODE, int NT, int MT, int DEPTH, int THREADS>
__global__ void __launch_bounds__(THREADS) w4_linear_kernel(W4Args a) {
    constexpr int TOK = kTokens<MODE>, P = kParts<MODE>;
    constexpr int kSize = MODE == kF32 ? 4 : MODE == kMx8 ? 1 : 2;
    extern __shared__ f32x4 sums[];  // [wavefronts][NT][64], a tile of columns at a time; then the staged columns
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, col = lane & 15;
    const int64_t tile0 = static_cast<int64_t>(blockIdx.x) * NT;
    const int64_t ntiles = a.w.tiles();
    const int steps = static_cast<int>(a.w.steps()), groups = static_cast<int>(a.w.groups());
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
    if (first >= last) return;
    const uint8_t *codes[NT], *scales[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int64_t tile = tile0 + i < ntiles ? tile0 + i : ntiles - 1;
        codes[i] = w + tile * steps * 1024;
        scales[i] = w + a.w.tile_codes() + tile * steps * 64;
    }
    // the row of x that position r of this workgroup's rows stands for
    const auto row_of = [&](int64_t r) -> int64_t {
        if (!a.slots) return r;
        const int64_t p = a.order[r];
        return p >= 0 && p < all ? p / a.slots : 0;
    };
    using S = Step<MODE, NT, MT>;
    const auto load_w = [&](S &s, int step) {
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            s.q[i] = *reinterpret_cast<const uint4 *>(codes[i] + static_cast<uint32_t>(step * 1024 + lane * 16));
            s.sw[i] = *reinterpret_cast<const uint32_t *>(scales[i] + static_cast<uint32_t>(step * 64 + col * 4));
        }
    };
    const int full = a.whole ? a.w.K / 128 : 0;  // steps whose inputs are all there, and aligned

    for (int64_t r0 = first; r0 < last; r0 += TOK * MT) {
        S ring[DEPTH];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (wave + d * waves < full) load_w(ring[d], wave + d * waves);
        // a direct type's lane owns a column of each tile, a row of x; columns past
        // the last row read it again, and nothing reads their sums
        const uint8_t *xrow[kStaged<MODE> ? TOK * MT : MT], *srow[MODE == kMx8 ? MT : 1];
        if constexpr (kStaged<MODE>) {
#pragma unroll
            for (int t = 0; t < TOK * MT; ++t)
                xrow[t] = static_cast<const uint8_t *>(a.x) + (r0 + t < last ? row_of(r0 + t) : 0) * a.ldx * kSize;
        } else {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int64_t at = r0 + m * TOK + col, r = row_of(at < last ? at : last - 1);
                xrow[m] = static_cast<const uint8_t *>(a.x) + r * a.ldx * kSize;
                if constexpr (MODE == kMx8) srow[m] = a.xs + r * a.ldxs;
            }
        }
        const auto load_x = [&](S &s, int step, auto whole) {
            constexpr bool kWhole = decltype(whole)::value;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if constexpr (kStaged<MODE>) {
                    constexpr int per = kWords<MODE> / TOK;
#pragma unroll
                    for (int t = 0; t < TOK; ++t)
                        if (r0 + m * TOK + t < last)
                            load_pair<MODE, kWhole>(s.x[m] + t * per, xrow[m * TOK + t], step * 128 + 2 * lane, a.w.K);
                } else {
                    load_column<MODE, kWhole>(s.x[m], xrow[m], step * 128 + 8 * g, a.w.K);
                }
                if constexpr (MODE == kMx8 && kWhole) {
                    s.sx[m] = *reinterpret_cast<const uint32_t *>(srow[m] + step * 4);
                } else if constexpr (MODE == kMx8) {
                    s.sx[m] = 0u;
                    for (int j = 0; j < 4; ++j)
                        if (step * 4 + j < groups) s.sx[m] |= static_cast<uint32_t>(srow[m][step * 4 + j]) << (8 * j);
                }
            }
        };
        f32x4 acc[NT][MT] = {};
        const auto multiply = [&](const S &s) {
            uint8_t *stage = nullptr;
            if constexpr (kStaged<MODE>) {
                // the wavefront's own columns: no other reads or writes them
                constexpr int per = kWords<MODE> / TOK;
                stage = reinterpret_cast<uint8_t *>(sums + waves * NT * 64) + wave * (MT * kStageTile);
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int t = 0; t < TOK; ++t)
                        if (r0 + m * TOK + t < last) {
                            const uint32_t *x = s.x[m] + t * per;
                            uint32_t parts[P];
                            if constexpr (MODE == kF32)
                                cut<P>(parts, __uint_as_float(x[0]), __uint_as_float(x[1]));
                            else
                                cut<P>(parts, F16::widen(x[0] & 0xffffu), F16::widen(x[0] >> 16));
#pragma unroll
                            for (int p = 0; p < P; ++p)
                                *reinterpret_cast<uint32_t *>(stage + m * kStageTile + (t * P + p) * kStageRow + lane * 4) =
                                    parts[p];
                        }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bf16x8 f[NT];
#pragma unroll
                for (int i = 0; i < NT; ++i)
                    f[i] = widen8(j == 0 ? s.q[i].x : j == 1 ? s.q[i].y : j == 2 ? s.q[i].z : s.q[i].w,
                                  scale_word(s.sw[i], j));
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    bf16x8 b;
                    if constexpr (kStaged<MODE>)
                        b = *reinterpret_cast<const bf16x8 *>(stage + m * kStageTile + col * kStageRow + (32 * j + 8 * g) * 2);
                    else
                        b = operand<MODE>(s.x[m] + j * (kWords<MODE> / 4), s.sx[MODE == kMx8 ? m : 0], j);
#pragma unroll
                    for (int i = 0; i < NT; ++i)
                        acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i], b, acc[i][m], 0, 0, 0);
                }
            }
        };
        // steps wave, wave + waves, ...: DEPTH of them loaded ahead; a last step
        // that is not full, and rows off 16-byte boundaries, value by value
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (wave + d * waves < full) load_x(ring[d], wave + d * waves, std::true_type{});
        for (int step = wave; step < full; step += DEPTH * waves) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                const int now = step + d * waves, next = now + DEPTH * waves;
                if (now < full) multiply(ring[d]);
                if (next < full) {
                    load_w(ring[d], next);
                    load_x(ring[d], next, std::true_type{});
                }
            }
        }
        for (int rest = full + (wave + waves - full % waves) % waves; rest < steps; rest += waves) {
            load_w(ring[0], rest);
            load_x(ring[0], rest, std::false_type{});
            multiply(ring[0]);
        }
        // add the wavefronts' sums up and the parts, and store
        const float *flat = reinterpret_cast<const float *>(sums);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            __syncthreads();  // what was there is stored
#pragma unroll
            for (int i = 0; i < NT; ++i) sums[(wave * NT + i) * 64 + lane] = acc[i][m];
            __syncthreads();
            for (int o = threadIdx.x; o < NT * TOK * 16; o += blockDim.x) {
                const int n = o & 15, t = (o >> 4) % TOK, i = (o >> 4) / TOK;
                const int64_t r = r0 + m * TOK + t, out = (tile0 + i) * 16 + n;
                if (r >= last || out >= a.w.N) continue;
                float v = 0.0f;
#pragma unroll
                for (int part = P - 1; part >= 0; --part) {
                    float u = 0.0f;
                    for (int z = 0; z < waves; ++z)
                        u += flat[((z * NT + i) * 64 + (n >> 2) * 16 + t * P + part) * 4 + (n & 3)];
                    v += u;
                }
                if (a.relu && v <= 0.0f) v = 0.0f;
                const int64_t p = a.slots ? a.order[r] : r;
                if (p >= 0 && p < all) store_as(a.y, p * a.ldy + out, v, a.ytype);
            }
        }
    }
}

template <int MODE, int NT, int MT, int DEPTH, int THREADS>
hipError_t run(const W4Args &a, int waves, hipStream_t s) {
    const int64_t tiles = (a.w.tiles() + NT - 1) / NT;
    const int64_t rows = kTokens<MODE> * MT;
    const unsigned y = static_cast<unsigned>(a.slots ? a.w.E + 1 : (a.T + rows - 1) / rows);
    if (waves > THREADS / 64) waves = THREADS / 64;
    const size_t lds = static_cast<size_t>(waves) * (sizeof(f32x4) * 64 * NT + (kStaged<MODE> ? MT * kStageTile : 0));
    w4_linear_kernel<MODE, NT, MT, DEPTH, THREADS>
        <<<dim3(static_cast<unsigned>(tiles), y), dim3(static_cast<unsigned>(64 * waves)), lds, s>>>(a);
    return hipGetLastError();
}

template <int MODE>
hipError_t by_tokens(const W4Args &a, hipStream_t s) {
    const int64_t rows = a.slots ? (static_cast<int64_t>(a.T) * a.slots + a.w.E - 1) / a.w.E : a.T;
    int waves = 1;
    while (waves < 8 && waves < a.w.steps()) waves *= 2;
    if constexpr (kStaged<MODE>) {
        if (rows <= kTokens<MODE>) return run<MODE, 1, 1, 4, 512>(a, waves, s);
        return run<MODE, 4, 2, 2, 256>(a, waves, s);
    } else {
        if (a.slots && rows <= kTokens<MODE>) return run<MODE, 1, 1, 2, 256>(a, waves, s);
        if (rows <= kTokens<MODE>) return run<MODE, 1, 1, 4, 512>(a, waves, s);
        if (rows <= 2 * kTokens<MODE>) return run<MODE, 2, 2, 2, 512>(a, waves, s);
        return run<MODE, 4, 4, 2, 256>(a, waves, s);
    }
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
