// Internal interface of LayerNorm for training (norm_train.cu).
#pragma once

#include "common.cuh"

namespace tbn {
namespace norm {

struct ForwardArgs {
    const void *x, *residual;
    int x_dtype, y_dtype;
    int64_t T;
    int32_t d;
    const float *gamma, *beta;
    float eps;
    void *sum, *y;
    float *mean, *rstd;
};
struct BackwardArgs {
    const void *dy, *x;
    int dy_dtype, x_dtype;
    int64_t T;
    int32_t d;
    const float *gamma, *mean, *rstd;
    const void *dsum;
    void *dx;
    float *dgamma, *dbeta;
};
size_t backward_workspace_bytes(int64_t T, int32_t d);
int forward(const ForwardArgs &a, cudaStream_t s);
int backward(const BackwardArgs &a, void *workspace, cudaStream_t s);

}  // namespace norm
}  // namespace tbn
