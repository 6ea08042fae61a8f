// Matrix products on the bf16 and fp16 matrix cores for operands that come as
// rows in memory: a tile of C[i][j] = sum over r of X(i, r) * W(j, r), both
// operands staged through LDS, for the experts' products, their gradients and
// the orthogonalisation.
//
//   - Either side may have its inner index r along the rows in memory (kAlong:
//     a row is one i or j) or across them (kAcross: a row is one r, as in a
//     product with a transposed matrix).  The second is turned over by the
//     transposing LDS read, so that no operand is ever transposed in memory.
//   - Rows may be picked by a list (a router's pairs by expert).
//   - 16-bit operands on 16-byte boundaries go into LDS by direct loads, others
//     through registers; chunks past an edge come from a block of zeros, or are
//     masked, so that nothing outside of an operand is read.
//   - fp32 operands are cut into three bf16 parts on their way into LDS, and six
//     of the nine products of parts are kept.  The others come to 2^-24 of a term
//     on average and to 2^-21 at most: fp32's precision at a sixth of the bf16
//     rate, which is 2.6 times that of the fp32 matrix instruction.
//
// 16 bits, v_mfma_f32_16x16x32: lane l holds 8 consecutive r (from 8 * (l / 16)) of
// row l % 16 of each operand; of the result, column l % 16 and the four rows from
// 4 * (l / 16) on.
// fp32's parts, v_mfma_f32_32x32x16: lane l holds 8 consecutive r (from 8 * (l / 32))
// of row l % 32 of each operand; of the result, column l % 32 and the rows
// 8 * (n / 4) + 4 * (l / 32) + n % 4.  W's rows are dealt to the instruction's so
// that these are the 16 consecutive j from 16 * (l / 32).
//
// LDS rows are whole multiples of the banks' width, so chunks of 16 bytes change
// places within a row by the row's number: the 64 lanes of a read meet all banks.
#pragma once

#include "ffn.hpp"

namespace isc {
namespace tp {

using f32x16 = __attribute__((ext_vector_type(16))) float;
using f32x4 = __attribute__((ext_vector_type(4))) float;
using s16x8 = __attribute__((ext_vector_type(8))) short;
using s16x4 = __attribute__((ext_vector_type(4))) short;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;

enum Side { kAlong, kAcross };

// A chunk past an edge comes from here.
static __device__ const uint4 kZeros[4] = {};

template <class T>
__device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    if constexpr (std::is_same_v<T, F16>)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
}

// 16 x 16 results of 32 inner indices.
template <class T>
__device__ __forceinline__ f32x4 mfma_16(s16x8 a, s16x8 b, f32x4 c) {
    if constexpr (std::is_same_v<T, F16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// A direct load into LDS: 16 bytes from each lane's address to `lds` (uniform)
// + 16 * lane.  In assembly because the compiler, which cannot tell the stages
// apart, would wait for it at the next transposing read; it has no output
// register, and land() waits for it before the barrier in front of its use.  The
// place is taken from m0, one wait state after it is written.
__device__ __forceinline__ void load_direct(const void *p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(lds) : "m0", "memory");
}

// This wavefront's loads have landed, all but the last N, and its LDS reads and writes
// are done; then all wavefronts'.
template <int N>
__device__ __forceinline__ void land() {
    static_assert(N >= 0 && N < 64, "vmcnt field");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

// This wavefront's LDS reads and writes are done; then all wavefronts'.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

__device__ __forceinline__ uint32_t lds_address(const void *p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void *)p));
}

// Eight values as they are in memory, the first n of them and zeros: a load whose widening
// can wait.
template <class T>
struct Raw8 {
    static constexpr bool kWide = sizeof(typename T::type) == 4;
    uint4 a, b;  // b: the upper four of 32-bit values
    __device__ __forceinline__ void load(const void *from, int n) {
        const char *p = static_cast<const char *>(from);
        if (n >= 8) {
            a = load_any<uint4>(p);
            if constexpr (kWide) b = load_any<uint4>(p + 16);
        } else if (n <= 0) {
            a = make_uint4(0, 0, 0, 0);
            if constexpr (kWide) b = a;
        } else if constexpr (kWide) {
            const auto one = [&](int i) { return i < n ? load_any<uint32_t>(p + 4 * i) : 0u; };
            a = make_uint4(one(0), one(1), one(2), one(3));
            b = make_uint4(one(4), one(5), one(6), one(7));
        } else {
            const auto two = [&](int i) {
                const uint32_t low = i < n ? load_any<uint16_t>(p + 2 * i) : 0u;
                return i + 1 < n ? low | static_cast<uint32_t>(load_any<uint16_t>(p + 2 * i + 2)) << 16 : low;
            };
            a = make_uint4(two(0), two(2), two(4), two(6));
        }
    }
    static __device__ __forceinline__ void widen2(float &low, float &high, uint32_t w) {
        low = T::widen(w & 0xffffu);
        high = T::widen(w >> 16);
    }
    __device__ __forceinline__ void widen(float (&f)[8]) const {
        if constexpr (kWide) {
            f[0] = __uint_as_float(a.x), f[1] = __uint_as_float(a.y), f[2] = __uint_as_float(a.z);
            f[3] = __uint_as_float(a.w), f[4] = __uint_as_float(b.x), f[5] = __uint_as_float(b.y);
            f[6] = __uint_as_float(b.z), f[7] = __uint_as_float(b.w);
        } else {
            widen2(f[0], f[1], a.x);
            widen2(f[2], f[3], a.y);
            widen2(f[4], f[5], a.z);
            widen2(f[6], f[7], a.w);
        }
    }
};

// One operand of a tile.  Rows of `width` elements, `stride` bytes apart.
struct Rows {
    const char *base;
    int64_t stride;
    const int32_t *list;  // row numbers (below 0: a row of zeros), or nullptr: 0, 1, 2, ...
    int count;            // rows there are
    int width;            // elements of a row
};

// Two fp32 values as three pairs of bf16 parts: the upper 16 bits, those of what is left,
// and of what that leaves.  Cut, not rounded, so that the largest values stay finite and
// 24 bits are all there.  Of a value that is not finite the second part is NaN.
__device__ __forceinline__ void cut(uint32_t v0, uint32_t v1, uint32_t &a, uint32_t &b, uint32_t &c) {
    const auto rest = [](uint32_t v) {
        return __float_as_uint(__uint_as_float(v) - __uint_as_float(v & 0xffff0000u));
    };
    const uint32_t r0 = rest(v0), r1 = rest(v1);
    a = __builtin_amdgcn_perm(v1, v0, 0x07060302u);  // the upper halves
    b = __builtin_amdgcn_perm(r1, r0, 0x07060302u);
    c = __builtin_amdgcn_perm(rest(r1), rest(r0), 0x07060302u);
}

// Stages of one operand: OUT outer indices (i or j) by BK inner ones.
// LISTED: rows across come by a list (rows along may have one or not).
template <class T, bool DIRECT, Side SIDE, bool LISTED, int OUT, int BK, int THREADS>
struct Stage {
    static constexpr bool kFetch = SIDE == kAcross && LISTED;
    static constexpr bool kWide = std::is_same_v<T, F32>;
    static constexpr int kParts = kWide ? 3 : 1;
    static constexpr int kSize = kWide ? 4 : 2;
    static constexpr int kRow = SIDE == kAlong ? BK / 8 : OUT / 8;  // chunks of 8 elements in an LDS row
    static constexpr int kLines = SIDE == kAlong ? OUT : BK;        // LDS rows
    static constexpr int kBytes = OUT * BK * 2;                     // of a part
    static constexpr int kLoads = kRow * kLines / THREADS;          // chunks of a thread
    static constexpr int kHop = THREADS / kRow;                     // LDS rows between a thread's chunks
    static_assert(kRow * kLines % THREADS == 0 && THREADS % kRow == 0 && kHop % (SIDE == kAcross ? 16 : 8) == 0,
                  "a thread's chunks");
    static_assert(!DIRECT || !kWide, "fp32 goes through registers");

    // Where chunk c of LDS row `line` is.  64 banks are 16 chunks: the 16 lanes that read a
    // chunk of consecutive rows, and the 32 that read four chunks of four rows, meet each once.
    static __device__ __forceinline__ int place(int line, int c) {
        constexpr int kShare = kRow < 16 ? 16 / kRow : 1;  // rows of all banks
        if constexpr (SIDE == kAcross)
            return c ^ (line / kShare % (4 / (kShare < 4 ? kShare : 4)) * 4) ^ (line >> 3 & 1) * 2;
        return c ^ (line / kShare % kRow);
    }

    const char *at[SIDE == kAlong ? kLoads : 1];  // kAlong: the rows' chunks at r = 0; else the first row's
    int width, count;                             // of `rows`, known to be uniform
    int64_t stride;
    bool edge;                                    // kAcross: some of the tile's columns are past the last one
    int32_t next[kFetch ? kLoads : 1];            // the listed rows of the stage to be sent
    int line, col;                                // this thread's first LDS row, and the element its chunks begin at
    Rows rows;
    Raw8<T> held[DIRECT ? 1 : kLoads];

    // o0: the tile's first outer index; inner: how many inner indices there are.
    __device__ __forceinline__ void begin(const Rows &r, int o0, int tid) {
        rows = r;
        width = __builtin_amdgcn_readfirstlane(r.width);
        count = __builtin_amdgcn_readfirstlane(r.count);
        stride = static_cast<int64_t>(static_cast<uint64_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(r.stride >> 32)))
                                          << 32 |
                                      static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(r.stride))));
        edge = o0 + OUT > width;
        line = tid / kRow;
        col = place(line, tid % kRow) * 8;
        if constexpr (SIDE == kAlong) {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                // a row past the last one takes the first one's place: its sums are not stored
                const int o = o0 + line + n * kHop;
                int64_t row = o < r.count ? o : 0;
                if (r.list) {
                    const int32_t listed = r.list[row];
                    row = listed < 0 ? 0 : listed;
                }
                at[n] = r.base + row * r.stride + int64_t{col} * kSize;
            }
        } else {
            col += o0;
            at[0] = r.base + int64_t{col} * kSize + (kFetch ? 0 : line * stride);
            if constexpr (kFetch) fetch(0, tid);
        }
    }

    // The listed rows of this thread's chunks of the stage from r0 on.  A wavefront's
    // loads take few rows each, whose numbers come by scalar loads: a vector load would
    // have to wait for every direct load sent before it.
    __device__ __forceinline__ void fetch(int r0, int tid) {
        constexpr int kRows = kRow < 64 ? 64 / kRow : 1;
        const int own = kRows > 1 ? (tid & 63) / kRow : 0;
        if (!rows.list) {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) next[n] = r0 + line + n * kHop < count ? r0 + line + n * kHop : -1;
            return;
        }
        const int first = r0 + __builtin_amdgcn_readfirstlane(line - own);
        using Scalar = const __attribute__((address_space(4))) int32_t *;
        Scalar list = reinterpret_cast<Scalar>(reinterpret_cast<uintptr_t>(rows.list));
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            int32_t row = -1;
#pragma unroll
            for (int q = 0; q < kRows; ++q) {
                const int r = first + n * kHop + q;
                const int32_t number = r >= count ? -1 : list[r];
                row = own == q ? number : row;
            }
            next[n] = row;
        }
    }

    // The address of chunk n of the stage at r0 ...
    __device__ __forceinline__ const char *chunk(int n, int r0) const {
        if constexpr (SIDE == kAlong)
            return at[n] + int64_t{r0} * kSize;
        else if constexpr (kFetch)
            // direct loads are taken where a stride has 32 bits (direct_rows): one instruction
            return at[0] + (DIRECT ? static_cast<int64_t>(uint64_t{static_cast<uint32_t>(next[n])} * static_cast<uint32_t>(stride))
                                   : next[n] * stride);
        else {
            int64_t past = (r0 + n * kHop) * stride;
            asm("" : "+s"(past));  // by the scalar unit: a vector one would multiply for every lane
            return at[0] + past;
        }
    }
    // ... and how many of its elements exist.
    __device__ __forceinline__ int there(int n, int r0) const {
        if constexpr (SIDE == kAlong)
            return width - r0 - col;
        else if constexpr (kFetch)
            return next[n] < 0 ? 0 : width - col;
        else
            return r0 + line + n * kHop < count ? width - col : 0;
    }

    // Sends load n of the stage from r0 on; a direct one to LDS at `lds`.
    __device__ __forceinline__ void send(int n, int r0, uint32_t lds, int wave) {
        const char *p = chunk(n, r0);
        if constexpr (DIRECT) {
            // width and column are multiples of 8: a chunk exists as a whole or not at all.  Where
            // all do, nothing is to be asked: the empty asm keeps this a branch.
            if (kFetch || (SIDE == kAlong ? r0 + BK > width : edge || r0 + BK > count)) {
                if constexpr (!kFetch) asm volatile("");
                p = there(n, r0) > 0 ? p : reinterpret_cast<const char *>(kZeros);
            }
            load_direct(p, lds + (n * THREADS + wave * 64) * 16);
        } else {
            held[n].load(p, there(n, r0));
        }
    }
    __device__ __forceinline__ void send_all(int r0, uint32_t lds, int wave, int tid) {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) send(n, r0, lds, wave);
        if constexpr (kFetch) fetch(r0 + BK, tid);
    }

    // Puts what the registers hold into LDS.
    __device__ __forceinline__ void commit(char *lds, int tid) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                char *to = lds + (n * THREADS + tid) * 16;
                if constexpr (!kWide) {
                    *reinterpret_cast<uint4 *>(to) = held[n].a;
                } else {
                    const uint32_t v[8] = {held[n].a.x, held[n].a.y, held[n].a.z, held[n].a.w,
                                           held[n].b.x, held[n].b.y, held[n].b.z, held[n].b.w};
                    uint32_t part[3][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        cut(v[2 * i], v[2 * i + 1], part[0][i], part[1][i], part[2][i]);
#pragma unroll
                    for (int q = 0; q < 3; ++q)
                        *reinterpret_cast<uint4 *>(to + q * kBytes) =
                            make_uint4(part[q][0], part[q][1], part[q][2], part[q][3]);
                }
            }
        }
    }

    // A matrix operand: 32 outer indices from o on, 16 inner ones from 16 * kk on.
    // DEALT: outer indices in the order that leaves a lane 16 consecutive results.
    template <bool DEALT>
    static __device__ __forceinline__ s16x8 operand(const char *lds, int o, int kk, int lane) {
        const int h = lane >> 5;
        if constexpr (SIDE == kAlong) {
            const int m = lane & 31;
            const int row = o + (DEALT ? 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3) : m);
            return *reinterpret_cast<const s16x8 *>(lds + (row * kRow + place(row, 2 * kk + h)) * 16);
        } else {
            // four rows of 16 outer indices a read and 16 lanes, each lane 4 of a row's
            const int i = lane & 15, u = 4 * ((lane >> 4) & 1) + (i & 3);
            const int c = o + 4 * (DEALT ? 4 * (u & 1) + (u >> 1) : u);
            s16x4 v[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int r = 16 * kk + 8 * h + 4 * q + (i >> 2);
                v[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(
                    lds + (r * kRow + place(r, c >> 3)) * 16 + (c & 7) * 2));
            }
            return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }

    // The same for mfma_16, of 32 inner indices from 32 * kk on and 16 outer ones, number t of
    // those of a wavefront, that begin at o: lane_at(o) + what t and kk change, which are bits
    // that the lane's place leaves alone or are flipped in it.
    static __device__ __forceinline__ int lane_at(int o, int lane) {
        const int i = lane & 15, g = lane >> 4;
        if constexpr (SIDE == kAlong) return ((o + i) * kRow + place(o + i, g)) * 16;
        const int r = 8 * g + (i >> 2), c = o + 4 * (i & 3);
        return (r * kRow + place(r, c >> 3)) * 16 + (c & 7) * 2;
    }
    static __device__ __forceinline__ s16x8 operand_16(const char *lds, int at, int t, int kk) {
        if constexpr (SIDE == kAlong) {
            return *reinterpret_cast<const s16x8 *>(lds + (at ^ 64 * kk) + t * 256 * kRow);
        } else {
            s16x4 v[2];
#pragma unroll
            for (int q = 0; q < 2; ++q)
                v[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(
                    lds + (at ^ 32 * t) + (32 * kk + 4 * q) * kRow * 16));
            return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// A workgroup's tile: BI x BJ results by WI x WJ wavefronts, BK inner indices a stage.
// Loads through registers have two stages in LDS.  Direct loads have two of W and three
// of X (160 KiB for 256 x 256, all of a compute unit's; 80 KiB for 128 x 128, so that
// two workgroups fit): X's have more than a stage's time to land, W's all of one.
//   256 x 256, eight wavefronts   a wavefront's 128 x 64 results take 12 operands for 32
//     products.  4096 tokens of 2048 through 8 of 64 experts of 1408, us a launch: 255 (740
//     TFLOP/s), by 128 x 128, whose rows fit the experts better, 259; dx of the same 260 and
//     337, dw 315 and 460.  Four wavefronts of 128 x 128 results, one a SIMD, are 15 %
//     slower, four stages of 32 inner indices 5 %, since half a line a row is asked for at
//     a time.
//   LISTED: whose rows across come by a list, X's 1, W's 2.
//   A stage of 256 x 256 takes 1.8 us with every compute unit busy; what is sent, read and
//     multiplied in it, without the tile around it, 1.4.
template <class T_, bool DIRECT_, Side XS, Side WS, int BI_, int BJ_, int WI_, int WJ_, int LISTED = 0,
          int BK_ = 64>
struct Tile {
    using T = T_;
    static constexpr bool DIRECT = DIRECT_, kXAcross = XS == kAcross;
    static constexpr int BI = BI_, BJ = BJ_, WI = WI_, WJ = WJ_;
    static constexpr int kWaves = WI * WJ, kThreads = 64 * kWaves;
    static constexpr int BK = std::is_same_v<T, F32> && BI > 64 ? 32 : BK_;
    // 16 bits go by the smaller instruction, which takes less power for a product.  Power is what
    // bounds a loop of nothing but a stage's products, reads and loads: with all compute
    // units busy 1.41 us on random operands, by 32 x 32 x 16 1.62, and 1.05 by that where all
    // operands are alike.
    static constexpr bool kSmall = !std::is_same_v<T, F32>;
    static constexpr int kEdge = kSmall ? 16 : 32;  // of an instruction's results
    static constexpr int FI = BI / WI / kEdge, FJ = BJ / WJ / kEdge;
    using Sums = std::conditional_t<kSmall, f32x4, f32x16>;
    using XStage = Stage<T, DIRECT, XS, (LISTED & 1) != 0, BI, BK, kThreads>;
    using WStage = Stage<T, DIRECT, WS, (LISTED & 2) != 0, BJ, BK, kThreads>;
    static constexpr int kParts = XStage::kParts;
    static constexpr int kXBytes = XStage::kBytes * kParts, kWBytes = WStage::kBytes * kParts;
    static constexpr int kXStages = DIRECT ? 3 : 2;
    static constexpr int kLds = kXStages * kXBytes + 2 * kWBytes;

    // fp32: the products with a part of less than the first add up beside the others, which
    // then are rounded once for every 16 inner indices, not six times.
    static constexpr int kSums = kParts > 1 ? 2 : 1;
    Sums acc[FJ][FI], low[kSums > 1 ? FJ : 1][kSums > 1 ? FI : 1];

    // What a wavefront multiplies at a time: 16 inner indices.
    struct Operands {
        s16x8 w[FJ][kParts], x[FI][kParts];
    };
    static constexpr int kReads = kParts * (FI + FJ);
    // Read n of a step's operands: those that the first products take come first.
    static __device__ __forceinline__ void read(Operands &o, int n, const char *x, const char *w, int kk, int wi, int wj,
                                                int lane) {
        const int p = kParts - 1 - n / (FI + FJ), f = n % (FI + FJ);
        if (f == 0 || f > FI)
            o.w[f == 0 ? 0 : f - FI][p] =
                WStage::template operand<true>(w + p * WStage::kBytes, wj + 32 * (f == 0 ? 0 : f - FI), kk, lane);
        else
            o.x[f - 1][p] = XStage::template operand<false>(x + p * XStage::kBytes, wi + 32 * (f - 1), kk, lane);
    }
    // between(n): what is issued behind product n, while the matrix cores have work.
    static constexpr int kProducts = FI * FJ * kParts * (kParts + 1) / 2;
    template <class Between>
    __device__ __forceinline__ void multiply(const Operands &o, Between &&between) {
        int n = 0;
#pragma unroll
        for (int sum = kParts - 1; sum >= 0; --sum)  // the small products first
#pragma unroll
            for (int p = 0; p <= sum; ++p)
#pragma unroll
                for (int j = 0; j < FJ; ++j)
#pragma unroll
                    for (int i = 0; i < FI; ++i) {
                        if (sum > 0)
                            low[j][i] = mfma<T>(o.w[j][p], o.x[i][sum - p], low[j][i]);
                        else
                            acc[j][i] = mfma<T>(o.w[j][p], o.x[i][sum - p], acc[j][i]);
                        between(n++);
                    }
    }

    // This wavefront's part of the tile.  A SIMD's two wavefronts (w and w + 4 of eight) have
    // neither rows nor columns in common, so that where a tile reaches past an edge the
    // ones that have nothing to do leave the matrix cores of every SIMD to the others.
    static __device__ __forceinline__ int part_i() {
        return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6)) / WJ * (BI / WI);
    }
    static __device__ __forceinline__ int part_j() {
        const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
        return (wave + (kWaves == 8 ? wave / WJ * (WJ / 2) : 0)) % WJ * (BJ / WJ);
    }

    // Where stages are in LDS.
    static __device__ __forceinline__ int w_at(int s) { return kXStages * kXBytes + (s & 1) * kWBytes; }
    static __device__ __forceinline__ int x_next(int at) { return at + kXBytes < kXStages * kXBytes ? at + kXBytes : 0; }

    XStage xs;
    WStage ws;

    // Sends the first loads of the tile at (i0, j0): direct ones of a stage of W and two of
    // X.  Nothing reads LDS any more when this is called, but for what each() puts into the
    // places that stay free.
    __device__ __forceinline__ void start(const Rows &x, const Rows &w, int i0, int j0, int inner, char *lds) {
        const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        if (inner <= 0) return;
        xs.begin(x, i0, tid);
        ws.begin(w, j0, tid);
        if constexpr (DIRECT) {
            const uint32_t base = lds_address(lds);
            xs.send_all(0, base, wave, tid);
            ws.send_all(0, base + w_at(0), wave, tid);
            if (inner > BK) xs.send_all(BK, base + kXBytes, wave, tid);
        }
    }

    // The sums of the tile that start() began, over `inner` inner indices, of whose rows and
    // columns the first `rows` and `cols` are asked for.  Operands are
    // read ahead of their products; a stage's last are in
    // registers when the wavefronts meet, so that behind the barrier its place is free.
    // Loads are sent one at a time between products: sent together they would hold the
    // wavefront, and the matrix cores with it, until the address unit has taken them.
    // landed: each() has waited for start()'s loads.
    __device__ __forceinline__ void sums(int inner, int rows, int cols, bool landed, char *lds) {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wi = part_i(), wj = part_j();
        const bool busy = wi < rows && wj < cols;
#pragma unroll
        for (int j = 0; j < FJ; ++j)
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int n = 0; n < kEdge * kEdge / 64; ++n) {
                    acc[j][i][n] = 0.0f;
                    if constexpr (kSums > 1) low[j][i][n] = 0.0f;
                }
        const int steps = (inner + BK - 1) / BK;
        if (steps <= 0) return;
        const uint32_t base = lds_address(lds);
        if constexpr (DIRECT) {
            if (landed)
                meet();
            else
                land<0>();
            if (steps > 1) ws.send_all(BK, base + w_at(1), wave, tid);
        } else {
            xs.send_all(0, base, wave, tid);
            ws.send_all(0, base, wave, tid);
            meet();
            xs.commit(lds, tid);
            ws.commit(lds + w_at(0), tid);
            land<0>();
        }
        if constexpr (kSmall)
            small_steps(steps, busy, wi, wj, lds);
        else
            wide_steps(steps, busy, wi, wj, lds);
        // no load into LDS may outlive its tile, and all of its reads are done before the next one's
        land<0>();
    }

    // fp32's stages
    __device__ __forceinline__ void wide_steps(int steps, bool busy, int wi, int wj, char *lds) {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        constexpr int kSteps16 = BK / 16;
        static_assert(kSmall || kSteps16 % 2 == 0, "a stage's first operands are always at[0]");
        int x_now = 0;  // the place in LDS of this stage's X
        Operands at[2];
#pragma unroll
        for (int n = 0; n < kReads; ++n) read(at[0], n, lds, lds + w_at(0), 0, wi, wj, lane);
        for (int s = 0; s < steps; ++s) {
            const bool more = s + 1 < steps;
            const int x_then = x_next(x_now);
            if (more) {
                xs.send_all((s + 1) * BK, 0, wave, tid);
                ws.send_all((s + 1) * BK, 0, wave, tid);
            }
#pragma unroll
            for (int kk = 0; kk < kSteps16; ++kk) {
                if (kk + 1 == kSteps16 && more) {
                    xs.commit(lds + x_then, tid);
                    ws.commit(lds + w_at(s + 1), tid);
                    land<0>();
                }
                // the operands of the next 16: behind the last stage's, those of some stage, which nothing takes
                const char *from_x = lds + (kk + 1 < kSteps16 ? x_now : x_then),
                           *from_w = lds + (kk + 1 < kSteps16 ? w_at(s) : w_at(s + 1));
                __builtin_amdgcn_sched_barrier(0);
                if (busy)
                    multiply(at[kk & 1], [&](int n) {
                        constexpr int kEach = (kReads + kProducts - 1) / kProducts;
#pragma unroll
                        for (int q = n * kEach; q < (n + 1) * kEach && q < kReads; ++q)
                            read(at[(kk + 1) & 1], q, from_x, from_w, (kk + 1) % kSteps16, wi, wj, lane);
                        __builtin_amdgcn_sched_barrier(0);
                    });
                __builtin_amdgcn_sched_barrier(0);
            }
            x_now = x_then;
        }
    }

    // 16 bits': a step of 32 inner indices is a product of each of X's operands, in turn, with
    // all of W's.  Of the 256 x 256 tile's X four are in registers, read three ahead of their
    // products, of smaller tiles' a step's beside the next one's; W's are a step's and the next.
    static constexpr int kAhead = FI > 4 ? 3 : FI, kPlaces = FI > 4 ? 4 : 2 * FI;
    static constexpr int kMeet = FI - kAhead;  // behind this many of X's operands only the next step's are read
    static_assert(!kSmall || FI <= 4 || (FI % 4 == 0 && DIRECT), "X's places");
    static constexpr int kWGroups = kAhead > 1 ? kAhead - 1 : 1, kWEach = (FJ + kWGroups - 1) / kWGroups;
    __device__ __forceinline__ void small_steps(int steps, bool busy, int wi, int wj, char *lds) {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const uint32_t base = lds_address(lds);
        constexpr int kSteps = BK / 32;
        static_assert(!kSmall || kSteps % 2 == 0, "a stage's first operands have the first places");
        int x_now = 0;  // the place in LDS of this stage's X
        const int lane_x = XStage::lane_at(wi, lane), lane_w = WStage::lane_at(wj, lane);
        s16x8 w[2][FJ], x[kPlaces];
        const auto at = [](int kk, int i) { return FI > 4 ? i % 4 : (kk & 1) * FI + i; };
#pragma unroll
        for (int j = 0; j < FJ; ++j) w[0][j] = WStage::operand_16(lds + w_at(0), lane_w, j, 0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) x[at(0, i)] = XStage::operand_16(lds, lane_x, i, 0);
        for (int s = 0; s < steps; ++s) {
            const bool more = s + 1 < steps, most = s + 2 < steps;
            const int x_then = x_next(x_now), x_last = x_next(x_then);
            if (!DIRECT && more) {
                xs.send_all((s + 1) * BK, 0, wave, tid);
                ws.send_all((s + 1) * BK, 0, wave, tid);
            }
#pragma unroll
            for (int kk = 0; kk < kSteps; ++kk) {
                const bool end = kk + 1 == kSteps;
                // behind the last stage's operands those of some stage are read, which nothing takes
                const char *from_x = lds + (end ? x_then : x_now), *from_w = lds + (end ? w_at(s + 1) : w_at(s));
                // X's next-but-two goes where the last stage's X was, W's next-but-one, from the
                // meeting on, where this stage's is
                const auto send = [&](int n) {
                    if constexpr (DIRECT) {
                        constexpr int kX = (XStage::kLoads + FI * FJ - 1) / (FI * FJ);
                        constexpr int kW = (WStage::kLoads + kAhead * FJ - 1) / (kAhead * FJ);
                        if (kk == 0 && most) {
#pragma unroll
                            for (int q = n * kX; q < (n + 1) * kX && q < XStage::kLoads; ++q) {
                                xs.send(q, (s + 2) * BK, base + x_last, wave);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                        }
                        const int m = n - kMeet * FJ;
                        if (end && most && m >= 0) {
#pragma unroll
                            for (int q = m * kW; q < (m + 1) * kW && q < WStage::kLoads; ++q) {
                                ws.send(q, (s + 2) * BK, base + w_at(s), wave);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                        }
                    }
                };
                const auto group = [&](int i) {
#pragma unroll
                    for (int j = 0; j < FJ; ++j) {
                        acc[j][i] = mfma_16<T>(w[kk & 1][j], x[at(kk, i)], acc[j][i]);
                        const int n = i - kMeet;  // W's of the next step, kWEach with each of X's
                        if (j == 0) {
                            const int t = i + kAhead;
                            if (t < FI)
                                x[at(kk, t)] = XStage::operand_16(lds + x_now, lane_x, t, kk);
                            else
                                x[at(kk + 1, t - FI)] = XStage::operand_16(from_x, lane_x, t - FI, (kk + 1) % kSteps);
                        }
                        if (n >= 0 && j < kWEach && n * kWEach + j < FJ)
                            w[(kk + 1) & 1][n * kWEach + j] =
                                WStage::operand_16(from_w, lane_w, n * kWEach + j, (kk + 1) % kSteps);
                        __builtin_amdgcn_sched_barrier(0);
                        send(i * FJ + j);
                    }
                };
                __builtin_amdgcn_sched_barrier(0);
                if (busy) {
#pragma unroll
                    for (int i = 0; i < kMeet; ++i) group(i);
                } else {
#pragma unroll
                    for (int n = 0; n < kMeet * FJ; ++n) send(n);
                }
                if (end && more) {
                    if constexpr (DIRECT) {
                        if (most)
                            land<DIRECT ? XStage::kLoads : 0>();
                        else
                            land<0>();
                    } else {
                        xs.commit(lds + x_then, tid);
                        ws.commit(lds + w_at(s + 1), tid);
                        land<0>();
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                if (busy) {
#pragma unroll
                    for (int i = kMeet; i < FI; ++i) group(i);
                } else {
#pragma unroll
                    for (int n = kMeet * FJ; n < FI * FJ; ++n) send(n);
                }
                if constexpr (DIRECT) {
                    if constexpr (WStage::kFetch) if (end && most) ws.fetch((s + 3) * BK, tid);
                    if constexpr (XStage::kFetch) if (kk == 0 && most) xs.fetch((s + 3) * BK, tid);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            x_now = x_then;
        }
    }

    // A wavefront's results pass through LDS, 32 rows at a time and in places that start()
    // leaves free, so that a row's columns are 8 consecutive ones of consecutive lanes:
    // stores are whole lines.  ahead(i, j): what out() reads beside the 8 results of row i
    // from column j on (of the tile's own numbering), sent for all of the 32 rows first;
    // out(i, j, v, ahead), which leaves in v what, if MIRROR, turned(j, i, v) gets of
    // column j, its 8 values from row i on.
    static constexpr int kCols = BJ / WJ, kChunks = kCols / 4, kLanes = kCols / 8;
    static constexpr int kScratch = 32 * kCols * 4;
    static_assert(!DIRECT || kWaves * kScratch <= kXBytes + kWBytes, "the places left free");
    static_assert(kWaves * kScratch <= kLds && kXBytes % kScratch == 0, "whole wavefronts' places");
    template <bool MIRROR, class Ahead, class Out, class Turned>
    __device__ __forceinline__ void each(char *lds, Ahead &&ahead, Out &&out, Turned &&turned) {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wi = part_i(), wj = part_j();
        char *own;
        if constexpr (DIRECT) {
            const int at = wave * kScratch;
            own = lds + (at < kXBytes ? 2 * kXBytes + at : 3 * kXBytes + kWBytes + at - kXBytes);
        } else {
            own = lds + wave * kScratch;
        }
        const auto place = [&](int row, int c) { return own + (row * kChunks + (c ^ (row & (kChunks - 1)))) * 16; };
#pragma unroll
        for (int i = 0; i < BI / WI / 32; ++i) {
            constexpr int kRows = 64 / kLanes;  // of all lanes at a time
            const int row = lane / kLanes, c = lane % kLanes * 2;
            decltype(ahead(0, 0)) beside[32 / kRows];
#pragma unroll
            for (int r = 0; r < 32 / kRows; ++r) beside[r] = ahead(wi + 32 * i + r * kRows + row, wj + 4 * c);
            if constexpr (kSums > 1)
#pragma unroll
                for (int j = 0; j < FJ; ++j) acc[j][i] += low[j][i];
            // the last rows' stores are the only ones that follow start()'s loads unwaited for
            if (i == BI / WI / 32 - 1) asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
#pragma unroll
            for (int j = 0; j < FJ; ++j)
                if constexpr (kSmall) {
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        *reinterpret_cast<float4 *>(place(16 * q + (lane & 15), 4 * j + (lane >> 4))) =
                            make_float4(acc[j][2 * i + q][0], acc[j][2 * i + q][1], acc[j][2 * i + q][2], acc[j][2 * i + q][3]);
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<float4 *>(place(lane & 31, 8 * j + 4 * (lane >> 5) + q)) = make_float4(
                            acc[j][i][4 * q], acc[j][i][4 * q + 1], acc[j][i][4 * q + 2], acc[j][i][4 * q + 3]);
                }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int r = 0; r < 32 / kRows; ++r) {
                const float4 a = *reinterpret_cast<const float4 *>(place(r * kRows + row, c));
                const float4 b = *reinterpret_cast<const float4 *>(place(r * kRows + row, c + 1));
                float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
                out(wi + 32 * i + r * kRows + row, wj + 4 * c, v, beside[r]);
                if constexpr (MIRROR) {
                    *reinterpret_cast<float4 *>(place(r * kRows + row, c)) = make_float4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<float4 *>(place(r * kRows + row, c + 1)) = make_float4(v[4], v[5], v[6], v[7]);
                }
            }
            if constexpr (MIRROR) {
                __builtin_amdgcn_wave_barrier();
#pragma unroll 1
                for (int r = 0; r < kCols; r += 16) {  // four lanes a column
                    const int col = r + lane / 4, from = lane % 4 * 8;
                    float v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        v[k] = reinterpret_cast<const float *>(place(from + k, col >> 2))[col & 3];
                    turned(wj + col, wi + 32 * i + from, v);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
};

// Tile `id` in the order of the launch: workgroups are dealt to the 8 XCDs in turn, and
// each XCD gets consecutive tiles, which share operands in its L2.
__device__ __forceinline__ int of_xcd(int id, int total) {
    const int each = total >> 3, more = total & 7, x = id & 7;
    return x * each + (x < more ? x : more) + (id >> 3);
}

// 8 values, or as many as there are places for, of a type known at run time.
__device__ __forceinline__ void store8_as(void *p, int64_t at, const float (&v)[8], int there, int type) {
    if (type == ISC_F32)
        store8<F32>(static_cast<float *>(p) + at, v, there);
    else if (type == ISC_BF16)
        store8<BF16>(static_cast<uint16_t *>(p) + at, v, there);
    else
        store8<F16>(static_cast<uint16_t *>(p) + at, v, there);
}

// Wavefronts that share a 128 x 128 tile's columns.  fp32 has eight in all: one of a SIMD's
// two cuts values while the other's products run (2048 tokens through 2 of 8 experts of
// 1408 of 2048, 232 us with four wavefronts, 187 with eight).
template <class T>
constexpr int kWavesOf128 = std::is_same_v<T, F32> ? 4 : 2;

// Inner indices of a stage of the experts' 64 x 64 tiles, of which there are few a compute
// unit: half as many meetings (300 tokens of 2048 through 2 of 4 experts of 1408 24.0 and 21.2 us
// by 64 and 128; where more workgroups share a compute unit, as in the orthogonalisation, 64).
template <bool DIRECT>
constexpr int kInner64 = DIRECT ? 128 : 64;

// The side of a launch's tiles, by how many of each there are (of 256, or 0 where they cannot
// be taken; of 128).  Half of the compute units busy on tiles of 256 beat all on smaller ones,
// which ask for twice the operands a product.  Where there are few tiles one's steps in turn
// are the time, and those of 64 x 64 are the shortest (us by 128 and by 64: 3 matrices of 777 x
// 1155, the whole call, 320 and 244; 777 tokens of 1155 through 2 of 7 experts of 515, fp32, 98
// and 47); fp32's tiles of 128 pay from fewer on, since one of them fills a compute unit (1024
// tokens of 2048 through 2 of 8 experts of 1408, 192 tiles: 109 and 145).
inline int tile_side(int64_t of256, int64_t of128, bool wide) {
    return of256 > 128 ? 256 : of128 > (wide ? 96 : 256) ? 128 : 64;
}

// Workgroups that fill the chip's 256 compute units: tiles beyond them are taken in turn,
// the next one's first loads on their way while a tile's results are stored.
template <class TL>
constexpr int kResident = 256 * (163840 / TL::kLds < 2 ? 1 : 163840 / TL::kLds < 4 ? 163840 / TL::kLds : 4);

// LDS of a kernel beyond 64 KiB has to be asked for, once for each device: the
// attribute belongs to the device's copy of the kernel.
template <auto *KERNEL>
hipError_t allow_lds(int bytes) {
    static uint64_t done = 0;  // a bit for each of the first 64 devices
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
    const uint64_t bit = dev < 64 ? uint64_t{1} << dev : 0;
    if (__atomic_load_n(&done, __ATOMIC_RELAXED) & bit) return hipSuccess;
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) __atomic_fetch_or(&done, bit, __ATOMIC_RELAXED);
    return e;
}

}  // namespace tp
}  // namespace isc
