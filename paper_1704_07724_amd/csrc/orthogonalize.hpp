// The orthogonalisation's launch (orthogonalize.hip).
#pragma once

#include "ffn.hpp"

namespace isc {

// The parts of its workspace, in bytes from its start.  State and operands have
// rows of np() elements, the square matrices of mp(), zeros behind the last column.
struct OrthShape {
    int B, M, N;
    __host__ __device__ bool wide() const { return M <= N; }
    __host__ __device__ int m() const { return wide() ? M : N; }
    __host__ __device__ int np() const { return (N + 7) / 8 * 8; }
    __host__ __device__ int mp() const { return (m() + 7) / 8 * 8; }
    __host__ __device__ int64_t of_state() const { return static_cast<int64_t>(M) * np(); }
    __host__ __device__ int64_t of_square() const { return static_cast<int64_t>(m()) * mp(); }
    __host__ __device__ static int64_t round(int64_t n) { return (n + 255) / 256 * 256; }
    __host__ __device__ int blocks() const {  // workgroups that sum a matrix's squares
        const int64_t n = (of_state() + 8191) / 8192;
        return static_cast<int>(n < 1024 ? n : 1024);
    }
    __host__ __device__ int64_t inverse() const { return round(8 * static_cast<int64_t>(B) * blocks()); }
    __host__ __device__ int64_t low() const { return inverse() + round(8 * static_cast<int64_t>(B)); }
    __host__ __device__ int64_t operand(int i) const { return low() + (1 + i) * round(2 * B * of_state()); }
    __host__ __device__ int64_t square(int i) const { return operand(2) + i * round(2 * B * of_square()); }
    // Matrices of which one side is at most 64 have all of A in a workgroup (orth_small.hip).
    __host__ __device__ bool small() const { return m() <= 64; }
    __host__ __device__ int64_t span() const { return wide() ? N : M; }  // the longer side
    // Parts in which A's sums over the longer side are made, and added up after: where A has so
    // few tiles that its inner indices in turn are the time.
    __host__ __device__ int parts() const {
        if (B < 1) return 1;  // an empty stack has no tiles to divide by
        if (small()) {
            const int64_t fours = (span() + 255) / 256;
            return static_cast<int>(fours < 16 ? fours : 16);
        }
        const int64_t side = (m() + 63) / 64, tiles = B * side * (side + 1) / 2, steps = (span() + 63) / 64;
        if (tiles > 64 || steps < 8) return 1;
        const int64_t most = 256 / tiles < steps / 2 ? 256 / tiles : steps / 2;
        return static_cast<int>(most < 16 ? most : 16);
    }
    int64_t partial() const { return square(2); }
    int64_t bytes() const {
        if (small()) return partial() + round(int64_t{2} * 4 * B * parts() * 4096);
        return partial() + (parts() > 1 ? round(4 * B * parts() * of_square()) : 0);
    }
};

struct OrthArgs {
    OrthShape s;
    const void *g;
    int64_t ldg;
    int type, otype, steps;
    const float *coef;  // host: three for each step
    float eps;
    void *o;
    int64_t ldo;
    char *ws;
};
bool orth_launches_fit(const OrthShape &s);
hipError_t launch_orthogonalize(const OrthArgs &a, hipStream_t s);
hipError_t launch_orth_norm(const OrthArgs &a, hipStream_t s);   // the parts of every |G|^2
hipError_t launch_orth_small(const OrthArgs &a, hipStream_t s);  // all of it, behind them

constexpr float kOrthUp = 64.0f;     // of every fp16 operand
constexpr float kOrthLow = 2048.0f;  // of what a state's operand leaves, beyond that

#if defined(__HIPCC__)
// 1 / (|G| + eps) of matrix n, from its parts' sums of squares, by all of a workgroup of 256 or
// 1024 threads; `sums` is its LDS.
__device__ __forceinline__ double orth_inverse_norm(const double *squares, int n, int blocks, float eps, double *sums) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < blocks; i += 256)
        if (threadIdx.x < 256) sum += squares[static_cast<int64_t>(n) * blocks + i];
    if (threadIdx.x < 256) sums[threadIdx.x] = sum;
    __syncthreads();
    for (int d = 128; d > 0; d /= 2) {
        if (threadIdx.x < static_cast<unsigned>(d)) sums[threadIdx.x] += sums[threadIdx.x + d];
        __syncthreads();
    }
    const double all = sums[0];
    __syncthreads();
    return 1.0 / (sqrt(all) + static_cast<double>(eps));
}
#endif

}  // namespace isc
