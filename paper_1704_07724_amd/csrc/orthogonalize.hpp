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
        const int64_t n = (of_state() + 16383) / 16384;
        return static_cast<int>(n < 256 ? n : 256);
    }
    __host__ __device__ int64_t low() const { return round(8 * static_cast<int64_t>(B) * blocks()); }
    __host__ __device__ int64_t operand(int i) const { return low() + (1 + i) * round(2 * B * of_state()); }
    __host__ __device__ int64_t square(int i) const { return operand(2) + i * round(2 * B * of_square()); }
    // Parts in which A's sums over the state's rows or columns are made, and added up after: where
    // A has so few tiles that its inner indices in turn are the time.
    int parts() const {
        const int64_t side = (m() + 63) / 64, tiles = B * side * (side + 1) / 2, steps = ((wide() ? N : M) + 63) / 64;
        if (tiles > 64 || steps < 8) return 1;
        const int64_t most = 256 / tiles < steps / 2 ? 256 / tiles : steps / 2;
        return static_cast<int>(most < 16 ? most : 16);
    }
    int64_t partial() const { return square(2); }
    int64_t bytes() const { return partial() + (parts() > 1 ? round(4 * B * parts() * of_square()) : 0); }
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

}  // namespace isc
