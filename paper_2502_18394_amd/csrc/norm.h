// Residual and norm: rows, and launchers of the kernels.
#pragma once
#include <hip/hip_runtime.h>

namespace spectre {

constexpr int kNormGroup = 128;                    // channels of a scale
constexpr int kNormChain = 128;                    // rows whose gradients a workgroup adds in 32 bits, at most
constexpr int kNormMostBytes = 32768;              // of a row

struct NormRows {                                  // row t at x + t * x_stride (elements)
    const void *x, *delta;                         // delta null: nothing is added
    long long x_stride, delta_stride;
    const float *w;                                // null: ones
    float eps;
    int T, D;
};
struct NormGrads {
    const void *dy, *dsum;                         // dsum null: none
    long long dy_stride, dsum_stride;
};

hipError_t load_kernels_norm();
hipError_t launch_norm(const NormRows &n, int io, void *sum, void *y, float *scales, hipStream_t st);     // scales: y in 8 bits
int norm_backward_blocks(int T, int groups, bool weights);   // with the weights' gradient: as many rows of partial sums
hipError_t launch_norm_backward(const NormRows &n, const NormGrads &g, int io, void *gx, float *gw, float *partial, hipStream_t st);

}  // namespace spectre
