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
//     of the nine products of parts are kept (the others are below 2^-24 of the
//     largest): fp32's precision at a sixth of the bf16 rate, which is 2.6 times
//     that of the fp32 matrix instruction.
//
// v_mfma_f32_32x32x16: lane l holds 8 consecutive r (from 8 * (l / 32)) of row
// l % 32 of each operand; of the result, column l % 32 and the rows
// 8 * (n / 4) + 4 * (l / 32) + n % 4.  W's rows are dealt to the instruction's so
// that these are the 16 consecutive j from 16 * (l / 32): a lane stores 32 or 64
// consecutive bytes.
//
// LDS rows are whole multiples of the banks' width, so chunks of 16 bytes change
// places within a row by the row's number: the 64 lanes of a read meet all banks.
#pragma once

#include "ffn.hpp"

namespace isc {
namespace tp {

using f32x16 = __attribute__((ext_vector_type(16))) float;
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

// A direct load into LDS: 16 bytes from each lane's address to `lds` (uniform)
// + 16 * lane.  In assembly because the compiler, which cannot tell the stages
// apart, would wait for it at the next transposing read; it has no output
// register, and land() waits for it before the barrier in front of its use.  The
// place is taken from m0, one wait state after it is written; m0 is left as it was.
__device__ __forceinline__ void load_direct(const void *p, uint32_t lds) {
    uint32_t kept;
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b32 m0, %0"
        : "=&s"(kept)
        : "v"(p), "s"(lds)
        : "memory");
}

// This wavefront's loads have landed and its LDS reads and writes are done; then all wavefronts'.
__device__ __forceinline__ void land() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ uint32_t lds_address(const void *p) {
    return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void *)p));
}

// One operand of a tile.  Rows of `width` elements, `stride` bytes apart.
struct Rows {
    const char *base;
    int64_t stride;
    const int32_t *list;  // row numbers (below 0: a row of zeros), or nullptr: 0, 1, 2, ...
    int count;            // rows there are
    int width;            // elements of a row
};

// fp32 values as three bf16 parts: the upper 16 bits, those of what is left, and
// of what that leaves.  Cut, not rounded, so that the largest values stay finite;
// a value that is not finite is its first part alone.
__device__ __forceinline__ void cut(float v, uint32_t &a, uint32_t &b, uint32_t &c) {
    const uint32_t u = __float_as_uint(v);
    a = u >> 16;
    const bool finite = (u & 0x7f800000u) != 0x7f800000u;
    if (!finite && (u & 0xffffu)) a |= 1u;  // a NaN whose upper bits are an infinity's
    const float r = finite ? v - __uint_as_float(u & 0xffff0000u) : 0.0f;
    const uint32_t ur = __float_as_uint(r);
    b = ur >> 16;
    c = BF16::narrow(r - __uint_as_float(ur & 0xffff0000u));
}

// Stages of one operand: OUT outer indices (i or j) by BK inner ones.
template <class T, bool DIRECT, Side SIDE, int OUT, int BK, int THREADS>
struct Stage {
    static constexpr bool kWide = std::is_same_v<T, F32>;
    static constexpr int kParts = kWide ? 3 : 1;
    static constexpr int kSize = kWide ? 4 : 2;
    static constexpr int kRow = SIDE == kAlong ? BK / 8 : OUT / 8;  // chunks of 8 elements in an LDS row
    static constexpr int kLines = SIDE == kAlong ? OUT : BK;        // LDS rows
    static constexpr int kBytes = OUT * BK * 2;                     // of a part
    static constexpr int kLoads = kRow * kLines / THREADS;          // chunks of a thread
    static constexpr int kHop = THREADS / kRow;                     // LDS rows between a thread's chunks
    static_assert(kRow * kLines % THREADS == 0 && THREADS % kRow == 0 && kHop % 8 == 0, "a thread's chunks");
    static_assert(!DIRECT || !kWide, "fp32 goes through registers");

    // Where chunk c of LDS row `line` is.
    static __device__ __forceinline__ int place(int line, int c) {
        if constexpr (SIDE == kAcross) return c ^ ((line & 3) << 1);
        return kRow == 8 ? c ^ (line & 7) : c ^ ((line >> 1) & 3);
    }

    const char *at[SIDE == kAlong ? kLoads : 1];  // kAlong: the rows' chunks at r = 0
    int32_t next[SIDE == kAcross ? kLoads : 1];   // kAcross: the rows of the next stage
    int line, col;                                // this thread's first LDS row, and the element its chunks begin at
    Rows rows;
    uint4 held[DIRECT ? 1 : kLoads][kWide ? 2 : 1];

    // o0: the tile's first outer index; inner: how many inner indices there are.
    __device__ __forceinline__ void begin(const Rows &r, int o0, int tid) {
        rows = r;
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
            at[0] = r.base + int64_t{col} * kSize;
            fetch(0);
        }
    }

    // kAcross: the row numbers of the stage from r0 on.
    __device__ __forceinline__ void fetch(int r0) {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int r = r0 + line + n * kHop;
            next[n] = r >= rows.count ? -1 : rows.list ? rows.list[r] : r;
        }
    }

    // The address of chunk n of the stage at r0, and how many of its elements exist.
    __device__ __forceinline__ const char *chunk(int n, int r0, int &there) const {
        if constexpr (SIDE == kAlong) {
            there = rows.width - r0 - col;
            return at[n] + int64_t{r0} * kSize;
        } else {
            there = next[n] < 0 ? 0 : rows.width - col;
            return at[0] + int64_t{next[n]} * rows.stride;
        }
    }

    static __device__ __forceinline__ void masked(uint4 (&v)[kWide ? 2 : 1], const char *p, int there) {
        uint32_t w[8];
        if constexpr (kWide) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = i < there ? load_any<uint32_t>(p + 4 * i) : 0u;
            v[0] = make_uint4(w[0], w[1], w[2], w[3]);
            v[1] = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = 2 * i < there ? load_any<uint16_t>(p + 4 * i) : 0u;
                if (2 * i + 1 < there) w[i] |= static_cast<uint32_t>(load_any<uint16_t>(p + 4 * i + 2)) << 16;
            }
            v[0] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }

    // Sends the loads of the stage from r0 on; direct ones to LDS at `lds`.
    __device__ __forceinline__ void issue(int r0, uint32_t lds, int wave) {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            int there;
            const char *p = chunk(n, r0, there);
            if constexpr (DIRECT) {
                // width and column are multiples of 8: a chunk exists as a whole or not at all
                load_direct(there > 0 ? p : reinterpret_cast<const char *>(kZeros), lds + (n * THREADS + wave * 64) * 16);
            } else if (there >= 8) {
                held[n][0] = load_any<uint4>(p);
                if constexpr (kWide) held[n][1] = load_any<uint4>(p + 16);
            } else {
                masked(held[n], p, there);
            }
        }
        if constexpr (SIDE == kAcross) fetch(r0 + BK);
    }

    // Puts what the registers hold into LDS.
    __device__ __forceinline__ void commit(char *lds, int tid) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                char *to = lds + (n * THREADS + tid) * 16;
                if constexpr (!kWide) {
                    *reinterpret_cast<uint4 *>(to) = held[n][0];
                } else {
                    const uint32_t v[8] = {held[n][0].x, held[n][0].y, held[n][0].z, held[n][0].w,
                                           held[n][1].x, held[n][1].y, held[n][1].z, held[n][1].w};
                    uint32_t part[3][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t a[2], b[2], c[2];
                        cut(__uint_as_float(v[2 * i]), a[0], b[0], c[0]);
                        cut(__uint_as_float(v[2 * i + 1]), a[1], b[1], c[1]);
                        part[0][i] = a[0] | a[1] << 16;
                        part[1][i] = b[0] | b[1] << 16;
                        part[2][i] = c[0] | c[1] << 16;
                    }
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
};

// A workgroup's tile: BI x BJ results by WI x WJ wavefronts, BK inner indices a
// stage, two stages in LDS.
template <class T_, bool DIRECT_, Side XS, Side WS, int BI_, int BJ_, int WI_, int WJ_>
struct Tile {
    using T = T_;
    static constexpr bool DIRECT = DIRECT_;
    static constexpr int BI = BI_, BJ = BJ_, WI = WI_, WJ = WJ_;
    static constexpr int kWaves = WI * WJ, kThreads = 64 * kWaves;
    static constexpr int BK = std::is_same_v<T, F32> ? 32 : 64;
    static constexpr int FI = BI / WI / 32, FJ = BJ / WJ / 32;
    using XStage = Stage<T, DIRECT, XS, BI, BK, kThreads>;
    using WStage = Stage<T, DIRECT, WS, BJ, BK, kThreads>;
    static constexpr int kParts = XStage::kParts;
    static constexpr int kXBytes = XStage::kBytes * kParts, kWBytes = WStage::kBytes * kParts;
    static constexpr int kLds = 2 * (kXBytes + kWBytes);

    f32x16 acc[FJ][FI];

    // Products of the stage at `x` and `w` in LDS.
    __device__ __forceinline__ void multiply(const char *x, const char *w, int wi, int wj, int lane) {
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk) {
            s16x8 a[FJ][kParts], b[FI][kParts];
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
#pragma unroll
                for (int f = 0; f < FJ; ++f)
                    a[f][p] = WStage::template operand<true>(w + p * WStage::kBytes, wj + 32 * f, kk, lane);
#pragma unroll
                for (int f = 0; f < FI; ++f)
                    b[f][p] = XStage::template operand<false>(x + p * XStage::kBytes, wi + 32 * f, kk, lane);
            }
#pragma unroll
            for (int sum = kParts - 1; sum >= 0; --sum)  // the small products first
#pragma unroll
                for (int p = 0; p <= sum; ++p)
#pragma unroll
                    for (int j = 0; j < FJ; ++j)
#pragma unroll
                        for (int i = 0; i < FI; ++i) acc[j][i] = mfma<T>(a[j][p], b[i][sum - p], acc[j][i]);
        }
    }

    // The sums of the tile at (i0, j0) over `inner` inner indices.
    __device__ __forceinline__ void run(const Rows &x, const Rows &w, int i0, int j0, int inner, char *lds) {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wi = wave / WJ * (BI / WI), wj = wave % WJ * (BJ / WJ);
#pragma unroll
        for (int j = 0; j < FJ; ++j)
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int n = 0; n < 16; ++n) acc[j][i][n] = 0.0f;
        const int steps = (inner + BK - 1) / BK;
        if (steps <= 0) return;
        XStage xs;
        WStage ws;
        xs.begin(x, i0, tid);
        ws.begin(w, j0, tid);
        const uint32_t base = lds_address(lds);
        xs.issue(0, base, wave);
        ws.issue(0, base + kXBytes, wave);
        xs.commit(lds, tid);
        ws.commit(lds + kXBytes, tid);
        land();
        for (int s = 0; s < steps; ++s) {
            const int now = (s & 1) * (kXBytes + kWBytes), then = (kXBytes + kWBytes) - now;
            if (s + 1 < steps) {
                xs.issue((s + 1) * BK, base + then, wave);
                ws.issue((s + 1) * BK, base + then + kXBytes, wave);
            }
            multiply(lds + now, lds + now + kXBytes, wi, wj, lane);
            if (s + 1 < steps) {
                xs.commit(lds + then, tid);
                ws.commit(lds + then + kXBytes, tid);
            }
            land();
        }
    }

    // out(f, i, j, v): 16 consecutive results of row i (this lane's f-th) from column j on, in
    // the tile's own numbering; all of a row's, before the next row.
    template <class Out>
    __device__ __forceinline__ void each(Out &&out) {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wi = wave / WJ * (BI / WI), wj = wave % WJ * (BJ / WJ);
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j)
                out(i, wi + 32 * i + (lane & 31), wj + 32 * j + 16 * (lane >> 5), acc[j][i]);
    }
};

// The tile that workgroup `id` of `total` takes: workgroups are dealt to the 8
// XCDs in turn, and each XCD gets consecutive tiles, which share operands in its L2.
__device__ __forceinline__ int of_xcd(int id, int total) {
    const int each = total >> 3, more = total & 7, x = id & 7;
    return x * each + (x < more ? x : more) + (id >> 3);
}

// 16 values to 16 or fewer places of a row.
template <class T>
__device__ __forceinline__ void store16(typename T::type *p, const f32x16 &v, int there) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = v[8 * q + i];
        if (there > 8 * q) store8<T>(p + 8 * q, u, there - 8 * q);
    }
}

// LDS of a kernel beyond 64 KiB has to be asked for, once for each device: the
// attribute belongs to the device's copy of the kernel.
template <class F>
hipError_t allow_lds(F *kernel, int bytes) {
    static uint64_t done = 0;  // a bit for each of the first 64 devices
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
    const uint64_t bit = dev < 64 ? uint64_t{1} << dev : 0;
    if (__atomic_load_n(&done, __ATOMIC_RELAXED) & bit) return hipSuccess;
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) __atomic_fetch_or(&done, bit, __ATOMIC_RELAXED);
    return e;
}

}  // namespace tp
}  // namespace isc
