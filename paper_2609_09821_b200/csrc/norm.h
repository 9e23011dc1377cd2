// Layer norm kernels: arguments and launchers.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "act8.cuh"

namespace im {

constexpr int kNormMaxCols = 8192;
constexpr int kNormMaxPartials = 592;      // rows of partial column sums that a workspace has room for at most; the backward pass writes one for
                                           // each of its CTAs, two an SM (296 rows on 148 SMs)

struct NormForward {
    const void *x;
    void *y;
    long long ldx, ldy;
    int M, N, relu;
    const float *gamma, *beta;             // or null: 1, 0
    float eps;
    float *mean, *rstd;                    // [M] or null
    Act8View keep;                         // code null: nothing is kept
};
struct NormBackward {
    const void *dy, *x;                    // x null: the normalised values come from `kept`
    void *dx;                              // or null
    long long ld_dy, ldx, ld_dx;
    int M, N, relu;
    const float *mean, *rstd, *gamma, *beta;
    Act8View kept;
    float *partial;                        // [gridDim.x][2][N] column sums of h xh and of h, or null
    float *dgamma, *dbeta;                 // [N] or null
    int finish;                            // > 0 (the launcher's): the grid is one cluster; the first `finish` CTAs have rows, all add up the sums
};

cudaError_t launch_norm_forward(const NormForward &a, int x_dtype, int y_dtype, int n_sm, cudaStream_t stream);
// *n_partials: the rows of a.partial that are still to be added up (0: dgamma and dbeta are done)
cudaError_t launch_norm_backward(const NormBackward &a, int x_dtype, int dy_dtype, int n_sm, int *n_partials, cudaStream_t stream);

}  // namespace im
