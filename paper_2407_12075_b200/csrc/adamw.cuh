// Internal interface of the optimizer step (adamw.cu).
#pragma once

#include "common.cuh"

namespace tbn {
namespace adamw {

constexpr int kBlock = 256;                 // elements that share a scale of 8-bit states: one warp, eight to a lane
constexpr int64_t kMost = (int64_t)1 << 42;  // elements of a tensor

struct Hyper {
    double lr, beta1, beta2, eps;
    int64_t step;
    const int64_t *step_dev;                // instead of step, or null
    const float *lr_dev;                    // instead of lr, or null
    const float *grad_scale;                // or null
    uint64_t seed;
};

size_t norm_workspace_bytes(int32_t count);
int launch_norm(const tbn_adamw_tensor *tensors, int32_t count, double max_norm, float *norm, float *scale, void *workspace,
                cudaStream_t s);
int launch_step(const tbn_adamw_tensor *tensors, int32_t count, const Hyper &h, cudaStream_t s);
int launch_unpack(const tbn_adamw_tensor *tensors, int32_t count, float *const *m, float *const *v, cudaStream_t s);

}  // namespace adamw
}  // namespace tbn
