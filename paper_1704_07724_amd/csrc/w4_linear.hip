// Products on 4-bit weights for a dense x: y[t][n] = sum_k w[n][k] x[t][k], by
// one matrix or by the experts that tokens were routed to.
//
// Both operands become bfloat16 without losing a bit, on the way from memory
// to the matrix cores: a weight has two significant bits and an 8-bit x four,
// each widened under its group's scale, two values an instruction; a 16- or
// 32-bit x is cut into parts of its next 8 significant bits (1 for bfloat16, 2
// for fp16, 3 for fp32).  Each part is a column of its own: the 16 columns of a
// matrix instruction hold 16, 8 or 5 tokens, and the parts' sums are added at
// the end, the small ones first.  Products are then exact and sums are fp32.  (Bits
// under 2^-133, bfloat16's smallest number, are lost: of fp32 inputs below 2^-110, and
// of 8-bit inputs under a scale byte below 3.  Weights have none.)
// (The scaled 8-bit matrix instruction would take both sides as they are
// stored, but it adds neighbouring products in fewer bits than fp32: 2^-6 next
// to 2^8 is lost.)
//
// A workgroup owns 16 NT outputs and MT tiles of columns; its wavefronts share
// the inputs, 128 at a time in turn, and their sums meet in LDS in the
// wavefronts' order, so a result does not depend on timing.  A wavefront holds
// DEPTH steps' operands in registers, loads in flight behind the matrix work.
//
// Few tokens are bound by reading the weights, 17/32 byte each: 64 experts of 1408
// outputs of 2048, 16 tokens 19.7 us, 4.4 TB/s; 4096 outputs of 9216, one fp32
// token 8.0 us, 2.5 TB/s, the start and the end of a launch the rest.  From some
// 40 tokens on what bounds it is x from the second cache, 16 to 64 columns for every
// workgroup, beside the matrix cores: 16384 outputs of 8192, 64 bfloat16 tokens
// 24.8 us (693 TFLOP/s), 2048 tokens 553 us (993 TFLOP/s).
#include "ffn.hpp"

#include <cstdint>
#include <type_traits>

namespace isc {
namespace {

using f32x4 = float __attribute__((ext_vector_type(4)));
using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

// How x is fed: from its rows as they stand, or (from kPacked on, one, two or
// three parts a value) as pack_x_kernel has laid its columns out.
constexpr int kMx8 = 0, kBf16 = 1, kF16 = 2, kF32 = 3, kPacked = 4;
template <int MODE>
constexpr int kParts = MODE >= kPacked ? MODE - kPacked + 1 : MODE == kF32 ? 3 : MODE == kF16 ? 2 : 1;
template <int MODE>
constexpr int kTokens = 16 / kParts<MODE>;
// 16- and 32-bit floats other than bfloat16 go through LDS, cut into parts once.
template <int MODE>
constexpr bool kStaged = MODE == kF16 || MODE == kF32;
// 32-bit words of a step's inputs that a lane loads: a column's 32 inputs as they
// stand, or for a staged type two neighbouring inputs of every token.
template <int MODE>
constexpr int kWords = MODE == kMx8 ? 8 : MODE == kF16 ? kTokens<kF16> : MODE == kF32 ? 2 * kTokens<kF32> : 16;
constexpr int kStageRow = 272;  // bytes of a staged column's 128 inputs; 16 spare spread the columns over the banks
constexpr int kStageTile = 16 * kStageRow;
constexpr int kSumTile = 4 * 17;  // a tile's sums, four outputs each, with a spare one a row for the banks

// One step's operands of a wavefront, as loaded.
template <int MODE, int NT, int MT>
struct Step {
    uint4 q[NT];
    uint32_t sw[NT];
    uint32_t x[MT][kWords<MODE>];
    uint32_t sx[MODE == kMx8 ? MT : 1];
};

// A column's inputs of one step: eight from 32 j + 8 g on for each j, k the
// first.  FULL: all of them are there.
template <int MODE, bool FULL>
__device__ __forceinline__ void load_column(uint32_t (&x)[kWords<MODE>], const uint8_t *row, int k, int K) {
    constexpr int per = kWords<MODE> / 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int at = k + 32 * j;
        if constexpr (FULL && MODE == kMx8) {
            const uint2 v = load_any<uint2>(row + at);
            x[j * per] = v.x;
            x[j * per + 1] = v.y;
        } else if constexpr (FULL) {
            const uint4 v = load_any<uint4>(row + 2 * at);
            x[j * per] = v.x;
            x[j * per + 1] = v.y;
            x[j * per + 2] = v.z;
            x[j * per + 3] = v.w;
        } else if (K >= 8) {
            // the eight before the row's end where these would pass it, moved to their places
            const int from = at < K - 8 ? at : K - 8, by = at - from;
            if constexpr (MODE == kMx8) {
                const uint64_t v = by < 8 ? load_any<uint64_t>(row + from) >> (8 * by) : 0u;
                x[j * per] = static_cast<uint32_t>(v);
                x[j * per + 1] = static_cast<uint32_t>(v >> 32);
            } else {
                const uint4 v = load_any<uint4>(row + 2 * from);
                uint32_t u[4] = {v.x, v.y, v.z, v.w};
                move_down(u, by);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[j * per + i] = u[i];
            }
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
template <int MODE, bool FULL>
__device__ __forceinline__ void load_pair(uint32_t *x, const uint8_t *row, int k, int K) {
    if constexpr (MODE == kF32) {
        const uint32_t *p = reinterpret_cast<const uint32_t *>(row) + k;
        if constexpr (FULL) {
            const uint2 v = load_any<uint2>(p);
            x[0] = v.x;
            x[1] = v.y;
        } else {
            x[0] = k < K ? p[0] : 0u;
            x[1] = k + 1 < K ? p[1] : 0u;
        }
    } else {
        const uint16_t *p = reinterpret_cast<const uint16_t *>(row) + k;
        if constexpr (FULL)
            x[0] = load_any<uint32_t>(p);
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
    if constexpr (MODE != kMx8) {
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

__device__ __forceinline__ uint32_t word_of(const uint4 &q, int j) {
    return j == 0 ? q.x : j == 1 ? q.y : j == 2 ? q.z : q.w;
}

// Four consecutive outputs, `n` of them there.
__device__ __forceinline__ void store4_as(void *y, int64_t at, const f32x4 &v, int64_t n, int type) {
    if (n < 4) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c < n) store_as(y, at + c, v[c], type);
    } else if (type == ISC_F32) {
        store_any(static_cast<float *>(y) + at, v);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = type == ISC_BF16 ? BF16::narrow(v[c]) : F16::narrow(v[c]);
        store_any(static_cast<uint16_t *>(y) + at, make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16));
    }
}

// REST: the inputs end within a step, for a type that is read as it stands.
template <int MODE, int NT, int MT, int DEPTH, int THREADS, bool REST>
__global__ void __launch_bounds__(THREADS) w4_linear_kernel(W4Args a) {
    constexpr int TOK = kTokens<MODE>, P = kParts<MODE>;
    constexpr int kSize = MODE == kF32 ? 4 : MODE == kMx8 ? 1 : 2;
    constexpr int ROUND = MT % 2 ? 1 : 2;  // tiles of columns whose sums are in LDS together
    extern __shared__ f32x4 sums[];         // [wavefronts][NT][ROUND][kSumTile]; then the staged columns
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
    const int full = MODE >= kPacked ? steps : a.w.K / 128;  // steps whose inputs are all there

    for (int64_t r0 = first; r0 < last; r0 += TOK * MT) {
        S ring[DEPTH];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)  // weights first: they wait for nothing
            if (full > wave) load_w(ring[d], wave + d * waves < full ? wave + d * waves : wave);
        // a direct type's lane owns a column of each tile, a row of x; columns past
        // the last row read it again, and nothing reads their sums
        const uint8_t *xrow[kStaged<MODE> ? TOK * MT : MT], *srow[MODE == kMx8 ? MT : 1];
        if constexpr (kStaged<MODE>) {
#pragma unroll
            for (int t = 0; t < TOK * MT; ++t)
                xrow[t] = static_cast<const uint8_t *>(a.x) + (r0 + t < last ? row_of(r0 + t) : 0) * a.ldx * kSize;
        } else if constexpr (MODE >= kPacked) {
            const int64_t tiles = (a.T + TOK - 1) / TOK;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int64_t tile = r0 / TOK + m;
                xrow[m] = a.columns + (tile < tiles ? tile : tiles - 1) * steps * 4096;
            }
        } else {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int64_t at = r0 + m * TOK + col, r = row_of(at < last ? at : last - 1);
                xrow[m] = static_cast<const uint8_t *>(a.x) + r * a.ldx * kSize;
                if constexpr (MODE == kMx8) srow[m] = a.xs + r * a.ldxs;
            }
        }
        const auto load_x = [&](S &s, int step, auto is_full) {
            constexpr bool kFull = decltype(is_full)::value;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                if constexpr (kStaged<MODE>) {
                    constexpr int per = kWords<MODE> / TOK;
#pragma unroll
                    for (int t = 0; t < TOK; ++t)
                        if (r0 + m * TOK + t < last)
                            load_pair<MODE, kFull>(s.x[m] + t * per, xrow[m * TOK + t], step * 128 + 2 * lane, a.w.K);
                } else if constexpr (MODE >= kPacked) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(
                            xrow[m] + static_cast<uint32_t>(step * 4096 + j * 1024 + lane * 16));
                        s.x[m][4 * j] = v.x;
                        s.x[m][4 * j + 1] = v.y;
                        s.x[m][4 * j + 2] = v.z;
                        s.x[m][4 * j + 3] = v.w;
                    }
                } else {
                    load_column<MODE, kFull>(s.x[m], xrow[m], step * 128 + 8 * g, a.w.K);
                }
                if constexpr (MODE == kMx8 && kFull) {
                    s.sx[m] = load_any<uint32_t>(srow[m] + step * 4);
                } else if constexpr (MODE == kMx8) {
                    uint32_t b[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) b[j] = srow[m][step * 4 + j < groups ? step * 4 + j : groups - 1];
                    s.sx[m] = 0u;
#pragma unroll
                    for (int j = 0; j < 4; ++j) s.sx[m] |= (step * 4 + j < groups ? b[j] : 0u) << (8 * j);
                }
            }
        };
        f32x4 acc[NT][MT] = {};
        bf16x8 w8[NT];  // the weights of a step's first word
        const auto multiply = [&](const S &s, const S &after) {
            uint8_t *stage = nullptr;
            if constexpr (kStaged<MODE>) {
                // the wavefront's own columns: no other reads or writes them
                constexpr int per = kWords<MODE> / TOK;
                stage = reinterpret_cast<uint8_t *>(sums + waves * NT * ROUND * kSumTile) + wave * (MT * kStageTile);
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
                // the next word's weights are widened between this word's products
                bf16x8 f[NT];
#pragma unroll
                for (int i = 0; i < NT; ++i) f[i] = w8[i];
                const S &from = j < 3 ? s : after;
#pragma unroll
                for (int i = 0; i < NT; ++i) w8[i] = widen8(word_of(from.q[i], (j + 1) & 3), scale_word(from.sw[i], (j + 1) & 3));
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
                if constexpr (MT * NT >= 4) {
#pragma unroll
                    for (int i = 0; i < MT * NT; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);              // a matrix instruction,
                        __builtin_amdgcn_sched_group_barrier(0x002, (24 + MT * NT - 1) / (MT * NT), 0);  // its share of the rest
                    }
                }
            }
        };
        const auto widen_first = [&](const S &s) {
#pragma unroll
            for (int i = 0; i < NT; ++i) w8[i] = widen8(s.q[i].x, scale_word(s.sw[i], 0));
        };
        // Such a step comes first, its loads in flight with the first ones of the others
        // (4096 outputs of 4064, one bfloat16 token: 5.0 us against 6.2 with the step at the
        // end and value by value).  A staged type's comes last: it has two values a lane
        // and a barrier before them.
        const bool has_rest = REST && full % waves == wave;
        S rest;
        if (has_rest) {
            load_w(rest, full);
            load_x(rest, full, std::false_type{});
        }
        // steps wave, wave + waves, ...: DEPTH of them loaded ahead, without a branch
        // around a load (past the last step it is loaded again), so that a wait
        // counts the loads behind it and leaves them in flight
        const int mine = full > wave ? (full - wave + waves - 1) / waves : 0;
        if (mine > 0) {
            const auto step_of = [&](int i) { return wave + (i < mine ? i : mine - 1) * waves; };
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) load_x(ring[d], step_of(d), std::true_type{});
            __builtin_amdgcn_sched_barrier(0);
            if (has_rest) {
                widen_first(rest);
                multiply(rest, rest);
            }
            if constexpr (DEPTH > 1) widen_first(ring[0]);
            int i = 0;
            for (; i + DEPTH <= mine; i += DEPTH) {
#pragma unroll
                for (int d = 0; d < DEPTH; ++d) {
                    // the ring's next step is there to widen from; a ring of one has just loaded it
                    if constexpr (DEPTH == 1) widen_first(ring[0]);
                    multiply(ring[d], ring[(d + 1) % DEPTH]);
                    const int next = step_of(i + d + DEPTH);
                    load_w(ring[d], next);
                    load_x(ring[d], next, std::true_type{});
                    __builtin_amdgcn_sched_barrier(0);  // the loads stay here, a ring ahead of their use
                }
            }
#pragma unroll
            for (int d = 0; d < DEPTH - 1; ++d)
                if (i + d < mine) multiply(ring[d], ring[d + 1]);
        } else if (has_rest) {
            widen_first(rest);
            multiply(rest, rest);
        }
        if constexpr (kStaged<MODE>)
            for (int step = full + (wave + waves - full % waves) % waves; step < steps; step += waves) {
                load_w(ring[0], step);
                load_x(ring[0], step, std::false_type{});
                widen_first(ring[0]);
                multiply(ring[0], ring[0]);
            }
        // add the wavefronts' sums up and the parts, and store: a thread four
        // outputs of a token, neighbouring threads neighbouring outputs
#pragma unroll
        for (int m0 = 0; m0 < MT; m0 += ROUND) {
            if (m0 > 0 || r0 > first) __syncthreads();  // what was there is stored
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int m = 0; m < ROUND; ++m)
                    sums[((wave * NT + i) * ROUND + m) * kSumTile + g * 17 + col] = acc[i][m0 + m];
            __syncthreads();
            for (int o = threadIdx.x; o < ROUND * TOK * NT * 4; o += blockDim.x) {
                const int quad = o % (NT * 4), t = o / (NT * 4) % TOK, m = o / (NT * 4) / TOK, i = quad >> 2;
                const int64_t r = r0 + (m0 + m) * TOK + t, out = tile0 * 16 + quad * 4;
                if (r >= last || out >= a.w.N) continue;
                f32x4 v = {};
#pragma unroll
                for (int part = P - 1; part >= 0; --part) {
                    f32x4 u = {};
                    for (int z = 0; z < waves; ++z)
                        u += sums[((z * NT + i) * ROUND + m) * kSumTile + (quad & 3) * 17 + t * P + part];
                    v += u;
                }
                if (a.relu)
#pragma unroll
                    for (int c = 0; c < 4; ++c) v[c] = v[c] <= 0.0f ? 0.0f : v[c];
                const int64_t p = a.slots ? a.order[r] : r;
                if (p >= 0 && p < all) store4_as(a.y, p * a.ldy + out, v, a.w.N - out, a.ytype);
            }
        }
    }
}

// x as matrix operands: for every tile of 16 columns, step of 128 inputs and
// word j of the weights' layout, 16 bytes a lane.  One thread each, and the next
// ones where there are more than a grid's; inputs past K are 0, so the product needs
// no last step of its own.
constexpr int64_t kPackBlocks = 1 << 16;  // workgroups of a grid, 4 KiB each at a time
template <int XTYPE>
__global__ void __launch_bounds__(256) pack_x_kernel(W4Args a) {
    constexpr int P = XTYPE == ISC_F32 ? 3 : XTYPE == ISC_F16 ? 2 : 1, TOK = 16 / P;
    const int64_t steps = a.w.steps(), tiles = (a.T + TOK - 1) / TOK;
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; item < tiles * steps * 256;
         item += static_cast<int64_t>(gridDim.x) * 256) {
        const int lane = static_cast<int>(item & 63), j = static_cast<int>(item >> 6 & 3);
        const int64_t tile = (item >> 8) / steps;
        const int step = static_cast<int>((item >> 8) % steps);
        const int col = lane & 15, k = step * 128 + j * 32 + (lane >> 4) * 8;
        const int64_t t = tile * TOK + col / P;
        uint32_t out[4] = {0u, 0u, 0u, 0u};
        const int n = t < a.T && col < TOK * P ? a.w.K - k : 0;
        if (n > 0) {
            if constexpr (XTYPE == ISC_MX8) {
                const uint8_t *p = static_cast<const uint8_t *>(a.x) + t * a.ldx + k;
                uint32_t v[2] = {0u, 0u};
                if (a.w.K >= 8) {  // (as load_column does)
                    const int by = n < 8 ? 8 - n : 0;
                    const uint64_t u = load_any<uint64_t>(p - by) >> (8 * by);
                    v[0] = static_cast<uint32_t>(u);
                    v[1] = static_cast<uint32_t>(u >> 32);
                } else {
                    for (int i = 0; i < 8; ++i)
                        if (i < n) v[i / 4] |= static_cast<uint32_t>(p[i]) << (8 * (i & 3));
                }
                const bf16x8 b = operand<kMx8>(v, a.xs[t * a.ldxs + k / 32], 0);
                const uint4 u = __builtin_bit_cast(uint4, b);
                out[0] = u.x, out[1] = u.y, out[2] = u.z, out[3] = u.w;
            } else {
                using T = std::conditional_t<XTYPE == ISC_F32, F32, std::conditional_t<XTYPE == ISC_F16, F16, BF16>>;
                float v[8];
                load8<T>(v, static_cast<const typename T::type *>(a.x) + t * a.ldx + k, n);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t parts[P];
                    cut<P>(parts, v[2 * i], v[2 * i + 1]);
                    out[i] = parts[0];
                    if (P > 1 && col % P == 1) out[i] = parts[P > 1 ? 1 : 0];
                    if (P > 2 && col % P == 2) out[i] = parts[P > 2 ? 2 : 0];
                }
            }
        }
        reinterpret_cast<uint4 *>(a.columns)[item] = make_uint4(out[0], out[1], out[2], out[3]);
    }
}

template <int MODE, int NT, int MT, int DEPTH, int THREADS>
hipError_t run(const W4Args &a, int waves, hipStream_t s) {
    const int64_t tiles = (a.w.tiles() + NT - 1) / NT;
    const int64_t rows = kTokens<MODE> * MT;
    const unsigned y = static_cast<unsigned>(a.slots ? a.w.E + 1 : (a.T + rows - 1) / rows);
    while (waves > 1 && waves / 2 >= a.w.steps()) waves /= 2;  // no more wavefronts than steps
    const size_t lds = static_cast<size_t>(waves) * (sizeof(f32x4) * kSumTile * NT * (MT % 2 ? 1 : 2) + (kStaged<MODE> ? MT * kStageTile : 0));
    const dim3 grid(static_cast<unsigned>(tiles), y), block(static_cast<unsigned>(64 * waves));
    if constexpr (MODE == kMx8 || MODE == kBf16)
        if (a.w.K % 128 != 0) {
            w4_linear_kernel<MODE, NT, MT, DEPTH, THREADS, true><<<grid, block, lds, s>>>(a);
            return hipGetLastError();
        }
    w4_linear_kernel<MODE, NT, MT, DEPTH, THREADS, false><<<grid, block, lds, s>>>(a);
    return hipGetLastError();
}

int parts_of(int xtype) { return xtype == ISC_F32 ? 3 : xtype == ISC_F16 ? 2 : 1; }

// Whether x is laid out first: where its columns fill more than one tile, and
// where reading them as they stand, row by row and for every workgroup, takes
// longer than the launch that lays them out: half a microsecond for a hundred
// columns and steps together, less where a workgroup has several tiles of outputs
// for them (us as they stand and laid out, bfloat16: 4096 outputs of 9216, 16
// tokens 12.7 and 10.3, 8 tokens 9.5 and 10.3; 300 of 16384, 8 tokens 13.0 and 11.7,
// 5 tokens 10.3 and 11.7; 5000 of 16384, 16 tokens 20.1 and 14.7, 8 tokens 14.8 and
// 14.6; 8192 of 32768, 16 tokens 40.8 and 40.0, 8 tokens 34 and 40).
bool packs(const W4Shape &w, int T, int xtype, int slots) {
    if (slots) return false;
    const int64_t columns = static_cast<int64_t>(T) * parts_of(xtype);
    return T > 16 / parts_of(xtype) || (w.tiles() <= 512 && columns >= (w.tiles() > 256 ? 12 : 6) && columns * w.steps() >= 1024);
}

// Tiles of outputs a wavefront keeps (NT), wavefronts that share the inputs and
// steps loaded ahead, by the workgroups there are to fill 256 compute units with;
// times in us, bfloat16 but where said.
//
// Up to 256 tiles of outputs: one each.  Four wavefronts a workgroup rather than
// eight (4096 x 4096, one token: 4.2 against 4.8), but for long rows and few tokens
// (4096 outputs of 9216, one token: 6.6 against 7.4).  Over 256 two, so that no
// compute unit gets a second workgroup after the first and x is read half as often;
// eight wavefronts where rows are long (8192 outputs of 32768, one token 29.6,
// 45.7 with four and 37.0 with one tile; of 2048 4.3 and 4.1).  Over 512 four
// tiles and eight wavefronts for the same reasons (11000 outputs of 8192, 16 tokens:
// 14.2 against 20.7), until two tiles and four wavefronts give every unit two
// workgroups, where tokens are few (16384 of 8192, one token: 12.9 against 14.1;
// 12000 of 11000: 16.5 against 15.9).  Over 1024 four tiles and four wavefronts
// (40000 of 2048, 16 tokens: 13.3 against 14.5 with eight and 16.3 with two
// tiles), with few tokens from 2048 on (24000 of 4096, one token: 11.3 against
// 10.8 with two tiles; 32768 of 3584 12.1 against 12.5).
//
// A staged x costs work for each step, less with more tiles: two from 256 tiles on
// (5000 outputs of 16384, 5 fp32 tokens: 19.9 against 25.4), four over 1024 (40000
// of 2048: 12.7 against 19.8).
//
// An expert has few rows and many experts run: four tiles, or two where tokens are
// few (64 experts of 1408 outputs of 2048: 16 tokens 18.6 against 20.4, one token
// 8.3 against 7.5), and three tiles of columns where an expert has 32 pairs on average
// (4096 tokens 545 against 685, 256 tokens 50.4 and 54.2; 128, 16 pairs, 39.0 and
// 34.3); of a staged type two, or four with many tokens and outputs (the
// same in fp32 with one, two and four: one token 16.2 9.3 9.7, 64 tokens 130 54.2
// 49.9; 8 experts of 1024 of 512, 100 tokens 16.0 14.3 15.8).
template <int MODE>
hipError_t rows_as_they_stand(const W4Args &a, hipStream_t s) {
    const int64_t tiles = a.w.tiles(), steps = a.w.steps();
    if constexpr (kStaged<MODE>) {
        if (a.slots)
            return a.T > 16 && tiles * a.w.E >= 1024 ? run<MODE, 4, 1, 1, 256>(a, 4, s) : run<MODE, 2, 1, 1, 256>(a, 4, s);
        if (tiles > 1024) return run<MODE, 4, 1, 1, 256>(a, 4, s);
        if (tiles > 256) return run<MODE, 2, 1, 2, 512>(a, 8, s);
        return run<MODE, 1, 1, 4, 512>(a, 8, s);
    } else {
        const bool few = a.T <= 4;
        if (a.slots && static_cast<int64_t>(a.T) * a.slots >= int64_t{32} * a.w.E) return run<MODE, 4, 3, 1, 256>(a, 4, s);
        if (a.slots) return few ? run<MODE, 2, 1, 2, 256>(a, 4, s) : run<MODE, 4, 1, 1, 256>(a, 4, s);
        if (tiles > 1024 && (!few || tiles >= 2048)) return run<MODE, 4, 1, 1, 256>(a, 4, s);
        if (tiles > 512 && tiles <= (few ? 896 : 1024)) return run<MODE, 4, 1, 1, 512>(a, 8, s);
        if (tiles > 512 || (tiles > 256 && steps < 32)) return run<MODE, 2, 1, 1, 256>(a, 4, s);
        if (tiles > 256) return run<MODE, 2, 1, 1, 512>(a, 8, s);
        if (steps > 48 && tiles >= 128 && few) return run<MODE, 1, 1, 2, 512>(a, 8, s);
        return run<MODE, 1, 1, 2, 256>(a, 4, s);
    }
}

// The same choice for an x that was laid out: of the shapes below, the one whose
// workgroups take the least time together.  With two steps ahead a compute unit
// holds one workgroup, with one step (fewer registers) two, which is better where
// there are more than 256; a round's time is what it measured (8192 inputs, 64
// bfloat16 tokens and more).  Small shapes fill the chip, large ones read less for
// each product.  Measured against the next best shape: 1024 outputs of 8192, 47
// tokens 9.2 us against 11.1; 4096 of 4096 at 64 tokens 9.6 (11.5) and at 130 14.0
// (16.0); 5000 of 16384 at 64 24.4 (28.8); 16384 of 8192 at 64 25.0 (27.4), at 130
// 50.2 (54.5), at 200 67.9 (73.2, and 78.7 with two steps ahead) and at 2048 549
// (599, 633), where 1000 TFLOP/s are done.
struct Shape {
    int nt, mt, depth;  // tiles of outputs and of columns a workgroup, steps ahead
    int round, rest;    // 0.1 us a round of 256 workgroups, of 512 with one step ahead; a last round of 256 of those
};
constexpr Shape kShapes[] = {{1, 1, 2, 95, 0},  {1, 2, 2, 123, 0}, {2, 2, 2, 140, 0},   {3, 2, 2, 160, 0},
                             {4, 2, 2, 186, 0}, {3, 3, 2, 190, 0}, {4, 3, 2, 207, 0},   {4, 4, 2, 235, 0},
                             {3, 3, 1, 245, 150}, {4, 3, 1, 285, 180}, {4, 4, 1, 360, 200}};
constexpr int64_t kGridRows = 65535;  // a launch's limit; four tiles of columns stay under it
constexpr int kShapeCount = sizeof(kShapes) / sizeof(kShapes[0]);

int64_t time_of(const Shape &h, int64_t workgroups) {
    if (h.depth == 2) return (workgroups + 255) / 256 * h.round;
    if (workgroups <= 256) return INT64_MAX;
    const int64_t left = workgroups % 512;
    return workgroups / 512 * h.round + (left > 256 ? h.round : left > 0 ? h.rest : 0);
}

template <int MODE, int I = 0>
hipError_t run_shape(int i, const W4Args &a, hipStream_t s) {
    if constexpr (I + 1 < kShapeCount)
        if (i != I) return run_shape<MODE, I + 1>(i, a, s);
    return run<MODE, kShapes[I].nt, kShapes[I].mt, kShapes[I].depth, 256>(a, 4, s);
}

template <int XTYPE>
hipError_t packed(const W4Args &a, hipStream_t s) {
    constexpr int P = XTYPE == ISC_F32 ? 3 : XTYPE == ISC_F16 ? 2 : 1, MODE = kPacked + P - 1;
    const int64_t tiles = (a.T + kTokens<MODE> - 1) / kTokens<MODE>;
    const int64_t blocks = tiles * a.w.steps();
    pack_x_kernel<XTYPE><<<dim3(static_cast<unsigned>(blocks < kPackBlocks ? blocks : kPackBlocks)), dim3(256), 0, s>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    // one tile of columns (long rows): two of outputs, as above (5000 outputs of
    // 16384: 14.7 us against 18.1 with one)
    if (tiles == 1 && a.w.tiles() > 256) return run<MODE, 2, 1, 1, 512>(a, 8, s);
    int best = 0;
    int64_t least = INT64_MAX;
    for (int i = 0; i < kShapeCount; ++i) {
        const Shape &h = kShapes[i];
        if ((tiles + h.mt - 1) / h.mt > kGridRows) continue;  // (a million fp32 tokens by three tiles)
        const int64_t time = time_of(h, ((a.w.tiles() + h.nt - 1) / h.nt) * ((tiles + h.mt - 1) / h.mt));
        if (time < least) least = time, best = i;
    }
    return run_shape<MODE>(best, a, s);
}

}  // namespace

size_t w4_linear_column_bytes(const W4Shape &w, int T, int xtype, int slots) {
    if (!packs(w, T, xtype, slots)) return 0;
    const int tokens = 16 / parts_of(xtype);
    return static_cast<size_t>((T + tokens - 1) / tokens) * static_cast<size_t>(w.steps()) * 4096;
}

hipError_t launch_w4_linear(const W4Args &a, hipStream_t s) {
    // a workgroup never spans more tokens than its tiles of columns hold, so one
    // tile is the limit of the rows as they stand
    const bool pack = packs(a.w, a.T, a.xtype, a.slots);
    switch (a.xtype) {
    case ISC_MX8: return pack ? packed<ISC_MX8>(a, s) : rows_as_they_stand<kMx8>(a, s);
    case ISC_BF16: return pack ? packed<ISC_BF16>(a, s) : rows_as_they_stand<kBf16>(a, s);
    case ISC_F16: return pack ? packed<ISC_F16>(a, s) : rows_as_they_stand<kF16>(a, s);
    default: return pack ? packed<ISC_F32>(a, s) : rows_as_they_stand<kF32>(a, s);
    }
}

}  // namespace isc
