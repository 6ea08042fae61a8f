// 4-bit weights: quantisation of fp32, fp16 or bf16 weights, and the two
// layouts that the products read (W4Shape).
//
// A code is a sign, two exponent bits and one mantissa bit (0, 0.5, 1, 1.5, 2,
// 3, 4, 6); 32 codes along an output's inputs share a power-of-two scale.
// Plain form: two codes a byte, the even input's in the low half, each output's
// row of ceil(K / 2) bytes after the other; scales ceil(K / 32) bytes a row.
//
// Done once for a matrix; memory bounds it.  8192 outputs of 32768 inputs, 285 MB
// in and out: tiles 95 us (3.0 TB/s), rows 121 us (2.4 TB/s), 57 us with the codes
// still in the last cache (244 us where each thread turned its own eight outputs
// over and read 32 bytes of a row at a time).
#include "ffn.hpp"

namespace isc {
namespace {

// One thread per group of 32 weights, and the next ones where there are more than a grid's.
constexpr int64_t kQuantizeBlocks = 1 << 22;
__global__ void __launch_bounds__(256) w4_quantize_kernel(const void *src, int type, int64_t ld, int64_t rows, int K,
                                                          uint8_t *codes, uint8_t *scales) {
    const int groups = (K + 31) / 32;
    for (int64_t item = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; item < rows * groups;
         item += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t row = item / groups;
        const int g = static_cast<int>(item % groups);
        const int n = K - g * 32 < 32 ? K - g * 32 : 32;
        uint32_t m = 0;
        for (int i = 0; i < n; ++i)
            m = op_max(m, __float_as_uint(load_as(src, row * ld + g * 32 + i, type)) & 0x7fffffffu);
        const uint32_t b = group_scale<2, 0x400000u>(m);  // 6 = 1.5 * 2^2
        scales[row * groups + g] = static_cast<uint8_t>(b);
        const float inv = __uint_as_float((254u - (b > 253u ? 253u : b)) << 23);
        uint8_t *out = codes + row * ((K + 1) / 2) + g * 16;
        for (int i = 0; i < n; i += 2) {
            // a group with a weight that is not finite is NaN by its scale: codes 0
            const float lo = b == 255u ? 0.0f : load_as(src, row * ld + g * 32 + i, type) * inv;
            const float hi = b == 255u || i + 1 >= n ? 0.0f : load_as(src, row * ld + g * 32 + i + 1, type) * inv;
            out[i / 2] = static_cast<uint8_t>(__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, lo, hi, 1.0f, 0));
        }
    }
}

__device__ __forceinline__ uint32_t code_of(const uint8_t *codes, int64_t row_bytes, int n, int k, int N, int K) {
    if (n >= N || k >= K) return 0u;
    const uint32_t b = codes[n * row_bytes + (k >> 1)];
    return k & 1 ? b >> 4 : b & 15u;
}

// tiles: one thread per 16 bytes of codes (four words of 8 inputs each) and, for
// 16 of 64 threads, the word of four scales.
__global__ void __launch_bounds__(256) w4_tiles_kernel(W4Shape w, const uint8_t *codes, const uint8_t *scales,
                                                       uint8_t *packed) {
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (item >= w.tiles() * w.steps() * 64) return;
    const int e = blockIdx.y;
    const int lane = static_cast<int>(item & 63);
    const int64_t block = item >> 6, step = block % w.steps(), tile = block / w.steps();
    const int n = static_cast<int>(tile * 16 + (lane & 15)), g = lane >> 4;
    const int k = static_cast<int>(step * 128 + g * 8);
    const int64_t rb = (w.K + 1) / 2, groups = w.groups();
    const uint8_t *src = codes + static_cast<int64_t>(e) * w.N * rb;
    uint8_t *dst = packed + static_cast<int64_t>(e) * w.tile_bytes();
    uint32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint8_t *at = src + n * rb + ((k + 32 * j) >> 1);
        v[j] = 0u;
        if (n < w.N && k + 32 * j + 8 <= w.K)
            v[j] = load_any<uint32_t>(at);
        else
            for (int i = 0; i < 8; ++i) v[j] |= code_of(src, rb, n, k + 32 * j + i, w.N, w.K) << (4 * i);
    }
    reinterpret_cast<uint4 *>(dst)[block * 64 + lane] = make_uint4(v[0], v[1], v[2], v[3]);
    if (g != 0) return;
    uint32_t s = 0u;
    for (int j = 0; j < 4; ++j) {
        const int64_t group = step * 4 + j;
        const uint32_t b = n < w.N && group < groups ? scales[(static_cast<int64_t>(e) * w.N + n) * groups + group] : 127u;
        s |= b << (8 * j);
    }
    reinterpret_cast<uint32_t *>(dst + w.tile_codes())[block * 16 + lane] = s;
}

// rows: a workgroup turns 128 outputs x 128 inputs over in LDS, so that either
// side's accesses are 64 bytes or more.
__global__ void __launch_bounds__(256) w4_rows_kernel(W4Shape w, const uint8_t *codes, const uint8_t *scales,
                                                      uint8_t *packed) {
    __shared__ uint32_t tile[128][17];  // an output's eights of inputs, and a spare word for the banks
    const int64_t np = w.np(), groups = w.groups(), across = np / 128;
    const int e = blockIdx.y;
    const int n0 = static_cast<int>(blockIdx.x % across) * 128;
    const int64_t g0 = blockIdx.x / across * 4;
    const int64_t rb = (w.K + 1) / 2;
    const uint8_t *src = codes + static_cast<int64_t>(e) * w.N * rb;
    uint8_t *dst = packed + static_cast<int64_t>(e) * w.row_bytes() + g0 * 17 * np;
    const int fast = threadIdx.x & 15, slow = threadIdx.x >> 4;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const int n = n0 + r * 16 + slow, k = static_cast<int>(g0 * 32) + fast * 8;
        const uint8_t *at = src + n * rb + (k >> 1);
        uint32_t v = 0u;
        if (n < w.N && k + 8 <= w.K)
            v = load_any<uint32_t>(at);
        else
            for (int j = 0; j < 8; ++j) v |= code_of(src, rb, n, k + j, w.N, w.K) << (4 * j);
        tile[r * 16 + slow][fast] = v;
    }
    __syncthreads();
    // eight outputs by eight inputs a thread
    const int g = slow >> 2, q = slow & 3;
    if (g0 + g < groups) {
        uint32_t in[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) in[i] = tile[fast * 8 + i][slow];
        uint8_t *rows = dst + g * 17 * np + np + n0 / 2;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t v = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) v |= (in[i] >> (4 * j) & 15u) << (4 * i);
            reinterpret_cast<uint32_t *>(rows + (q * 8 + j) * (np / 2))[fast] = v;
        }
    }
    for (int i = threadIdx.x; i < 512; i += 256) {
        const int n = n0 + (i & 127), at = i >> 7;
        if (g0 + at < groups)
            dst[at * 17 * np + n] = n < w.N ? scales[(static_cast<int64_t>(e) * w.N + n) * groups + g0 + at] : 127;
    }
}

unsigned blocks_for(int64_t items) { return static_cast<unsigned>((items + 255) / 256); }

}  // namespace

hipError_t launch_w4_quantize(const W4Shape &w, const void *src, int type, int64_t ld, uint8_t *codes, uint8_t *scales,
                              hipStream_t s) {
    const int64_t rows = static_cast<int64_t>(w.E) * w.N;
    const int64_t blocks = (rows * w.groups() + 255) / 256;
    w4_quantize_kernel<<<dim3(static_cast<unsigned>(blocks < kQuantizeBlocks ? blocks : kQuantizeBlocks)), dim3(256), 0, s>>>(
        src, type, ld, rows, w.K, codes, scales);
    return hipGetLastError();
}

hipError_t launch_w4_pack(const W4Shape &w, int layout, const uint8_t *codes, const uint8_t *scales, uint8_t *packed,
                          hipStream_t s) {
    if (layout == ISC_W4_TILES) {
        const dim3 grid(blocks_for(w.tiles() * w.steps() * 64), static_cast<unsigned>(w.E));
        w4_tiles_kernel<<<grid, dim3(256), 0, s>>>(w, codes, scales, packed);
    } else {
        const dim3 grid(static_cast<unsigned>(w.np() / 128 * ((w.groups() + 3) / 4)), static_cast<unsigned>(w.E));
        w4_rows_kernel<<<grid, dim3(256), 0, s>>>(w, codes, scales, packed);
    }
    return hipGetLastError();
}

}  // namespace isc
