// Internal interface between the two translation units of the head losses: head_loss.cu (labels, packing, reductions,
// orchestration) and tc_head.cu (the tcgen05 contractions).
#pragma once

#include "common.cuh"

namespace tbn {

int *device_status_ptr();                  // the current device's status record (api.cu); null on error

namespace head {

constexpr int kTile = 256;                 // tokens x classes of one output tile (two CTAs, 128 rows each)
constexpr int kMaxSplits = 16;

__host__ __device__ inline int64_t round_up64(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

// What the epilogues need to know about one kept token row.
struct __align__(16) RowInfo {
    float lse2;                            // log2 of the row's sum of exponentials (backward)
    float g;                               // dloss (backward)
    int32_t label;                         // cross entropy: the target class
    int32_t row;                           // the row's index in the caller's tensors
};

#ifdef __CUDACC__
// The factor in [1, 2) that the bf16 form takes out of the gradient's tokens before dz is rounded and puts back into the sums:
// the mantissa of the first kept token's g that has one (of the first 32, so that the look is short: tokens of weight 0 at
// the front are common, a whole warp of them is not).  Under a mean every token has the same g; with it in dz the largest
// entry of every row, -g (1 - q), would be rounded the same way, and all of dx and dw off by up to 2^-8 with it.
__device__ __forceinline__ float common_mantissa(const RowInfo *rows, int32_t n_live)
{
    for (int32_t i = 0; i < n_live && i < 32; ++i) {
        const uint32_t b = __float_as_uint(rows[i].g), e = b & 0x7f800000u;
        if (e != 0u && e != 0x7f800000u) return __uint_as_float((b & 0x007fffffu) | 0x3f800000u);
    }
    return 1.0f;
}
#endif

// A bf16 (one plane) or fp32 (three bf16 planes: the value's first, second and third eight bits) operand as the contractions read it.
struct Operand {
    const void *data;
    int64_t rows, plane_rows;              // rows that exist, rows between two planes
    int32_t cols, ld;                      // columns that exist, row pitch in elements (a multiple of 8)
};

// Which tokens take part.
struct Labels {
    const int64_t *target;                 // cross entropy
    int64_t ignore_index;
    int32_t V;
    const uint8_t *flags;                  // distillation: written by teacher_kernel
    __device__ __forceinline__ bool live(int64_t t) const {
        if (flags) return flags[t] != 0;
        const int64_t c = target[t];
        return c != ignore_index && c >= 0 && c < V;
    }
};

int sm_count();

struct LogitsArgs {                        // logits of all kept tokens against classes [v0, v0 + width)
    Operand x, w;
    int32_t w_row0;                        // w's row of class v0 (0 where w is packed for one piece at a time)
    int planes;
    const int32_t *n_live;                 // null: the T rows in their own order (forward)
    const RowInfo *rows;                   // null with n_live
    Labels labels;                         // used without rows
    int32_t bn;                            // classes of a tile: a multiple of 32 up to 256 (backward: of 32 per epilogue warp)
    const float *bias;                     // V or null
    float scale2;                          // log2(e) / tau
    int64_t T, Tpad;
    int32_t v0, width;
    const int2 *list;                      // distillation: [T][K] (class, probability), ascending, INT32_MAX behind the last; else null
    const uint16_t *list_start;            // [T][pitch]: where the units + 1 units of classes begin in a row's list
    int32_t K, unit, units, pitch;
    // forward: (maximum, sum, dot, unused) of every token and epilogue warp's classes (bn / 2): [Tpad][parts]
    float4 *part;
    int32_t parts;
    // backward
    void *dz;                              // [planes][ldz / 64][Tpad][64], see tc_head.cu
    int32_t ldz;
    float *col_part;                       // [Tpad / 32][ldz] or null
    int *status;
};
int launch_head_stats(const LogitsArgs &a, cudaStream_t s);
int launch_head_dz(const LogitsArgs &a, cudaStream_t s);

struct GradArgs {                          // dX (+)= dz W, dW = dz^T X for one piece of the vocabulary
    Operand x, w;
    int32_t w_row0;                        // as in LogitsArgs
    int planes;
    const int32_t *n_live;
    const RowInfo *rows;
    float tau;                             // what the sums over dz are multiplied by
    const void *dz;
    int64_t T, Tpad;
    int32_t d, v0, width, ldz;
    bool want_dx, want_dw;
    // dX: into `dx` by row when no slots are used, else fp32 partial sums [split][Tpad][slot_ld], added to when `dx_add`
    void *dx;
    int dx_bf16;
    float *dx_slots;
    int32_t dx_splits;
    int dx_add, dx_last;                   // dx_last: this piece is the last one (without splits it finishes dx)
    // dW: rows v0 .. of `dw`, or fp32 partial sums [split][round_up(width, 256)][slot_ld]
    void *dw;
    int dw_bf16;
    float *dw_slots;
    int32_t dw_splits;
    int32_t slot_ld;                       // d in whole panels of 64
    int *status;
};
int launch_head_grads(const GradArgs &a, cudaStream_t s);


// One call of either loss, as the C entry points hand it over.
struct HeadCall {
    const void *x, *w;
    int dtype;                             // of x and w
    int64_t T;
    int32_t d, V;
    const float *bias;
    const int64_t *targets;                // cross entropy
    int64_t ignore_index;
    const int64_t *top_index;              // distillation: K > 0
    const void *top_logit;
    int top_dtype;
    int32_t K;
    float tau;
    float *loss_out, *lse_out;             // forward
    const float *lse, *dloss;              // backward
    void *dx, *dw;
    int dx_dtype, dw_dtype;
    float *db;
};
constexpr int32_t kMaxListed = 1024;
size_t workspace_bytes(int64_t T, int32_t d, int32_t V, int dtype, int32_t K, bool backward);
int forward(const HeadCall &c, void *workspace, size_t workspace_bytes, cudaStream_t s);
int backward(const HeadCall &c, void *workspace, size_t workspace_bytes, cudaStream_t s);

}  // namespace head
}  // namespace tbn
