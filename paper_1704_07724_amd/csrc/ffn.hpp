// Shared by the feed-forward operators (norm, routing, products on 4-bit
// weights): element types, wavefront reductions, the 8-bit and 4-bit group
// formats, and the launchers behind the C entry points in ffn_api.hip.
#pragma once

#include "isc_internal.hpp"

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>

namespace isc {

// --- element types ----------------------------------------------------------

struct F32 {
    using type = float;
    static __device__ __forceinline__ float load(const float *p) { return *p; }
};
struct F16 {
    using type = uint16_t;
    static __device__ __forceinline__ float widen(uint32_t b) {
        return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(b)));
    }
    static __device__ __forceinline__ uint32_t narrow(float v) {
        // the fp32 value, rounded: not folded into the instruction that made it, whose
        // one rounding would give another last bit from kernel to kernel
        asm("" : "+v"(v));
        return __builtin_bit_cast(uint16_t, static_cast<_Float16>(v));
    }
    static __device__ __forceinline__ float load(const uint16_t *p) { return widen(*p); }
};
struct BF16 {
    using type = uint16_t;
    static __device__ __forceinline__ float widen(uint32_t b) { return __uint_as_float(b << 16); }
    // to nearest, ties to even; a NaN stays one (the compiler's conversion)
    static __device__ __forceinline__ uint32_t narrow(float v) {
        return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
    }
    static __device__ __forceinline__ float load(const uint16_t *p) { return widen(*p); }
};

template <class T>
__device__ __forceinline__ void store(typename T::type *p, float v) {
    if constexpr (sizeof(typename T::type) == 4)
        *p = v;
    else
        *p = static_cast<uint16_t>(T::narrow(v));
}

// One value of a type known at run time.
__device__ __forceinline__ float load_as(const void *p, int64_t i, int type) {
    if (type == ISC_F32) return static_cast<const float *>(p)[i];
    const uint32_t b = static_cast<const uint16_t *>(p)[i];
    return type == ISC_BF16 ? BF16::widen(b) : F16::widen(b);
}
__device__ __forceinline__ void store_as(void *p, int64_t i, float v, int type) {
    if (type == ISC_F32)
        static_cast<float *>(p)[i] = v;
    else
        static_cast<uint16_t *>(p)[i] = static_cast<uint16_t>(type == ISC_BF16 ? BF16::narrow(v) : F16::narrow(v));
}

// Wide accesses at any address: the memory path takes a vector access at the
// alignment of its elements and below, so rows need not start on 16 bytes.
template <class V>
__device__ __forceinline__ V load_any(const void *p) {
    V v;
    __builtin_memcpy(&v, p, sizeof(V));
    return v;
}
template <class V>
__device__ __forceinline__ void store_any(void *p, const V &v) {
    __builtin_memcpy(p, &v, sizeof(V));
}

// Eight 16-bit values moved down by `by` of them, 0 from above.
__device__ __forceinline__ void move_down(uint32_t (&w)[4], int by) {
    uint32_t w0 = w[0], w1 = w[1], w2 = w[2], w3 = w[3];
    if (by & 4) w0 = w2, w1 = w3, w2 = 0u, w3 = 0u;
    if (by & 2) w0 = w1, w1 = w2, w2 = w3, w3 = 0u;
    const uint32_t half = by & 1 ? 16 : 0, all = by < 8 ? 0xffffffffu : 0u;
    w[0] = __builtin_amdgcn_alignbit(w1, w0, half) & all;
    w[1] = __builtin_amdgcn_alignbit(w2, w1, half) & all;
    w[2] = __builtin_amdgcn_alignbit(w3, w2, half) & all;
    w[3] = __builtin_amdgcn_alignbit(0u, w3, half) & all;
}

// Eight consecutive values, or the first n of them and zeros.
template <class T>
__device__ __forceinline__ void load8(float (&v)[8], const typename T::type *p, int n) {
    if (n >= 8) {
        if constexpr (sizeof(typename T::type) == 4) {
            const float4 a = load_any<float4>(p), b = load_any<float4>(p + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = load_any<uint4>(p);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = T::widen(w[i] & 0xffffu);
                v[2 * i + 1] = T::widen(w[i] >> 16);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? T::load(p + i) : 0.0f;
}
template <class T>
__device__ __forceinline__ void store8(typename T::type *p, const float (&v)[8], int n) {
    if (n >= 8) {
        if constexpr (sizeof(typename T::type) == 4) {
            store_any(p, make_float4(v[0], v[1], v[2], v[3]));
            store_any(p + 4, make_float4(v[4], v[5], v[6], v[7]));
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = T::narrow(v[2 * i]) | T::narrow(v[2 * i + 1]) << 16;
            store_any(p, make_uint4(w[0], w[1], w[2], w[3]));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) store<T>(p + i, v[i]);
}

// --- wavefront reductions by data-parallel moves ----------------------------
// Each step takes the other operand from a lane of the same row of 16, then
// from the row before, so no LDS round trip is paid; every lane gets lane
// 63's total.

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp(uint32_t old, uint32_t v) {
    return static_cast<uint32_t>(
        __builtin_amdgcn_update_dpp(static_cast<int>(old), static_cast<int>(v), CTRL, ROWS, 0xf, false));
}
#define ISC_WAVE_REDUCE(v, ident, op)                              \
    v = op(v, dpp<0x111, 0xf>(ident, v)); /* row_shr:1 */          \
    v = op(v, dpp<0x112, 0xf>(ident, v)); /* row_shr:2 */          \
    v = op(v, dpp<0x114, 0xf>(ident, v)); /* row_shr:4 */          \
    v = op(v, dpp<0x118, 0xf>(ident, v)); /* row_shr:8 */          \
    v = op(v, dpp<0x142, 0xa>(ident, v)); /* row_bcast:15 */       \
    v = op(v, dpp<0x143, 0xc>(ident, v)); /* row_bcast:31 */       \
    return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), 63))

__device__ __forceinline__ uint32_t op_max(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t op_min(uint32_t a, uint32_t b) { return a < b ? a : b; }
__device__ __forceinline__ uint32_t op_sum(uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) { ISC_WAVE_REDUCE(v, 0u, op_max); }
__device__ __forceinline__ uint32_t wave_min(uint32_t v) { ISC_WAVE_REDUCE(v, 0xffffffffu, op_min); }
__device__ __forceinline__ uint32_t wave_sum_bits(uint32_t v) { ISC_WAVE_REDUCE(v, 0u, op_sum); }
#undef ISC_WAVE_REDUCE
__device__ __forceinline__ float wave_sum(float v) { return __uint_as_float(wave_sum_bits(__float_as_uint(v))); }

// The same within rows of 16 lanes: every lane gets its row's, the same in all
// of them (each step adds or compares what the two sides hold alike).
#define ISC_ROW_REDUCE(v, op)                           \
    v = op(v, dpp<0xb1, 0xf>(v, v));  /* quad_perm 1,0,3,2 */ \
    v = op(v, dpp<0x4e, 0xf>(v, v));  /* quad_perm 2,3,0,1 */ \
    v = op(v, dpp<0x141, 0xf>(v, v)); /* row_half_mirror */   \
    v = op(v, dpp<0x140, 0xf>(v, v)); /* row_mirror */        \
    return v
__device__ __forceinline__ uint32_t row_max(uint32_t v) { ISC_ROW_REDUCE(v, op_max); }
__device__ __forceinline__ uint32_t row_min(uint32_t v) { ISC_ROW_REDUCE(v, op_min); }
__device__ __forceinline__ uint32_t row_sum_bits(uint32_t v) { ISC_ROW_REDUCE(v, op_sum); }
#undef ISC_ROW_REDUCE
__device__ __forceinline__ float row_sum(float v) { return __uint_as_float(row_sum_bits(__float_as_uint(v))); }

// An unsigned order of floats: a > b as numbers exactly when order(a) > order(b)
// (NaN aside; -0 orders below +0, so a caller ranks v + 0.0f).
__device__ __forceinline__ uint32_t order(float v) {
    const uint32_t b = __float_as_uint(v);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unorder(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

// --- group formats ----------------------------------------------------------
// A scale is one byte b and stands for 2^(b - 127); 255 stands for NaN.

// The scale byte of a group whose largest magnitude has the bits `abits`:
// the smallest power of two that brings it to `top` or below, where
// top = (1 + TOPM / 2^23) 2^TOPE.  255 where the magnitude is not finite.
template <int TOPE, uint32_t TOPM>
__device__ __forceinline__ uint32_t group_scale(uint32_t abits) {
    if (abits >= 0x7f800000u) return 255u;
    const int e = static_cast<int>(abits >> 23) - TOPE + ((abits & 0x7fffffu) > TOPM ? 1 : 0);
    return static_cast<uint32_t>(e > 0 ? e : 0);
}

// --- launchers --------------------------------------------------------------

// Threads that a launch may have along a dimension of its grid: fewer than 2^32.
// Calls of more rows than that take are launched in parts.
constexpr int64_t kLaunchThreads = (int64_t{1} << 32) - 1;

// `bytes` past p, which may be none.
template <class P>
P *past(P *p, int64_t bytes) {
    return p ? reinterpret_cast<P *>(reinterpret_cast<uintptr_t>(p) + static_cast<uintptr_t>(bytes)) : nullptr;
}

struct NormArgs {
    const void *x, *r, *w;      // r: nullptr without a residual
    void *h, *y, *q, *scales;   // each nullptr where it is not asked for
    float *rstd;
    int64_t ldx, ldr, ldh, ldy, ldq, lds;
    int T, D, type, wtype;
    float eps;
};
hipError_t launch_rmsnorm(const NormArgs &a, hipStream_t s);

struct NormBwdArgs {
    const void *dy, *h, *w, *dh;  // dh: nullptr without a second gradient
    const float *rstd;
    void *dx;
    float *dw, *part;  // part: norm_bwd_blocks() rows of D sums
    int64_t ldy, ldh, ldd, ldx;
    int T, D, type, wtype;
};
int norm_bwd_blocks(int T, int D);
hipError_t launch_rmsnorm_bwd(const NormBwdArgs &a, hipStream_t s);

struct RouteArgs {
    const void *logits;
    const float *bias;  // nullptr: none
    int64_t ld;
    int T, E, k, type, sigmoid, groups, keep, renorm;
    float scale;
    int32_t *ids;
    float *weights;
    int32_t *offsets, *order;  // both nullptr where the lists are not asked for
    uint16_t *counts;          // a row of counts for every workgroup, where there are several
};
size_t route_count_bytes(int T, int E);
hipError_t launch_route(const RouteArgs &a, hipStream_t s);

struct RouteBwdArgs {
    const float *dweights;
    const void *logits;
    const int32_t *ids;
    void *dlogits;
    int64_t ld, ldd;
    int T, E, k, type, sigmoid, renorm;
    float scale;
};
hipError_t launch_route_bwd(const RouteBwdArgs &a, hipStream_t s);

// 4-bit weights of E matrices N x K in one of two layouts.
//   tiles: for every 16 outputs and 128 inputs one KiB, lane l of a wavefront
//     owning 16 bytes: output l % 16, and in word j the inputs 32 j + 8 (l / 16)
//     .. + 8, in order; so a lane's word is a matrix operand of 32 inputs, one
//     group.  The scales of such a step, a word for each of the 16 outputs,
//     follow after all codes of the matrix.
//   rows: for every 32 inputs the outputs' scales (Np bytes), then 32 rows of
//     Np / 2 bytes, one per input, outputs in order (Np: N up to 128s); so the
//     weights of one input are contiguous, as the convolution's filters are.
struct W4Shape {
    int E, N, K;
    __host__ __device__ int64_t tiles() const { return (N + 15) / 16; }
    __host__ __device__ int64_t steps() const { return (K + 127) / 128; }
    __host__ __device__ int64_t tile_codes() const { return tiles() * steps() * 1024; }
    __host__ __device__ int64_t tile_bytes() const { return tile_codes() + tiles() * steps() * 64; }
    __host__ __device__ int64_t np() const { return (N + 127) / 128 * 128; }
    __host__ __device__ int64_t groups() const { return (K + 31) / 32; }
    __host__ __device__ int64_t row_bytes() const { return groups() * 17 * np(); }
    int64_t bytes(int layout) const { return E * (layout == ISC_W4_TILES ? tile_bytes() : row_bytes()); }
};
hipError_t launch_w4_quantize(const W4Shape &w, const void *src, int type, int64_t ld, uint8_t *codes,
                              uint8_t *scales, hipStream_t s);
hipError_t launch_w4_pack(const W4Shape &w, int layout, const uint8_t *codes, const uint8_t *scales, uint8_t *packed,
                          hipStream_t s);

struct W4Args {
    W4Shape w;
    const uint8_t *packed;
    const void *x;
    const uint8_t *xs;  // the scales of an 8-bit x
    int64_t ldx, ldxs, ldy;
    int T, slots, xtype, ytype, relu;  // slots 0: one matrix, no experts
    const int32_t *ids, *offsets, *order;
    const float *weights;
    void *y;
    float *part;
    uint8_t *columns;  // w4_linear_column_bytes() of room for x as matrix operands
};
size_t w4_linear_column_bytes(const W4Shape &w, int T, int xtype, int slots);
hipError_t launch_w4_linear(const W4Args &a, hipStream_t s);
// Ranges that the skipping product's inputs are cut into (each a row of sums
// in `part` where there are several).
int w4_skip_ranges(const W4Shape &w, int T, int slots);
hipError_t launch_w4_skip(const W4Args &a, hipStream_t s);

// The current device's check of the C entry points (isc_api.hip).
int require_gfx950();

}  // namespace isc
