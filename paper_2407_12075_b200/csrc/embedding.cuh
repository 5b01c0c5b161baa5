// Internal interface of the embedding lookup and its gradient (embedding.cu).
#pragma once

#include "common.cuh"

namespace tbn {
namespace embed {

struct LookupArgs {
    const int64_t *ids;
    int64_t T;
    int32_t d, V;
    int64_t padding;                        // an id that counts as outside the vocabulary
    float scale;
    const void *table;                      // V x d, or null with a tiled table
    int table_dtype;
    const uint32_t *tile;
    int64_t q;
    const float *alpha;
    int per_tile;
    void *y;
    int y_dtype;
};
struct GradArgs {
    const int64_t *ids;
    int64_t T;
    int32_t d, V;
    int64_t padding;
    float scale;
    const void *dy;
    int dy_dtype;
    void *dw;
    int dw_dtype;
    int add;                                // to what dw holds, instead of overwriting it
};
int lookup(const LookupArgs &a, cudaStream_t s);
size_t gradient_workspace_bytes(int64_t T, int32_t d, int32_t V);
int gradient(const GradArgs &a, void *workspace, cudaStream_t s);

}  // namespace embed
}  // namespace tbn
