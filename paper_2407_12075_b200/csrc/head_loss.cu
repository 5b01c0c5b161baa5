// Losses of a large-vocabulary head: labels, operand packing, reductions and the order of the launches.  The
// contractions are in tc_head.cu.
//
//   z_tv = x_t . w_v + b_v;  lse_t = log sum_v exp(z_tv / tau)
//   cross entropy (tau = 1)   loss_t = lse_t - z_t,label
//   distillation              loss_t = tau^2 sum_j p_tj (log p_tj - z_t,idx(t,j) / tau + lse_t)
//   gradient                  dz_tv = dloss_t tau (exp(z_tv / tau - lse_t) - sum_{j: idx(t,j) = v} p_tj)
//                             (held without tau, which the sums over it are multiplied by: it may be anything from 1e-30 to 1e30)
//
// Cross entropy is distillation from one entry of probability 1, so both share every kernel; only where the entries come
// from differs.  The logits are never stored: the forward keeps one (maximum, sum, weighted dot) record of 16 bytes per token
// and 128 classes (64 with fp32 operands, fewer in narrow tiles), the backward recomputes the logits piece by piece of the
// vocabulary and stores dz for one piece at a time.
//
// Tokens that are left out (ignored targets, empty teacher rows) are dropped first: the kept rows are packed to the front,
// so no kernel computes anything for the others and nothing in their rows -- infinities, NaN -- can reach a result.
#include <climits>

#include "head_loss.cuh"

namespace tbn {
namespace head {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr size_t kPieceBytes = (size_t)256 << 20;      // bound on one piece of dz (a piece has at least 1024 classes)

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// ---- the teacher's entries ---------------------------------------------------------------------------
// One warp per token: p = softmax(logit / tau) over the entries whose index is a class and whose logit is above
// -infinity, sum p log p, and the entries sorted by class (by position among equals), which is the order in which the
// epilogues meet the classes.
constexpr int kMaxUnits = 2046;                        // of a list_start row: 4 KB per warp
inline int teacher_warps(int32_t Kp) { return Kp <= 512 ? 4 : 2; }
inline size_t teacher_smem(int32_t Kp, int32_t pitch) { return (size_t)Kp * 12 + (size_t)pitch * 2; }      // per warp

template <typename TL>
__global__ void __launch_bounds__(128)
teacher_kernel(const int64_t *__restrict__ index, const TL *__restrict__ logit, int64_t T, int32_t K, int32_t Kp, int32_t V,
               float inv_tau, int32_t unit, int32_t units, int32_t pitch, int2 *__restrict__ list, uint16_t *__restrict__ list_start,
               uint8_t *__restrict__ flags, float2 *__restrict__ stats)
{
    extern __shared__ __align__(16) uint8_t teacher_mem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int warps = blockDim.x >> 5;
    uint64_t *key = reinterpret_cast<uint64_t *>(teacher_mem) + (size_t)warp * Kp;
    float *prob = reinterpret_cast<float *>(reinterpret_cast<uint64_t *>(teacher_mem) + (size_t)warps * Kp) + (size_t)warp * Kp;
    uint16_t *start = reinterpret_cast<uint16_t *>(teacher_mem + (size_t)warps * Kp * 12) + (size_t)warp * pitch;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t t = (int64_t)blockIdx.x * warps + warp;
    if (t >= T) return;
    float top = -INFINITY;
    bool any = false, nan = false;
#pragma unroll 4
    for (int32_t j = lane; j < Kp; j += 32) {
        const int64_t c = j < K ? index[t * K + j] : -1;
        float l = j < K ? load_as_float(logit, t * K + j) : 0.0f;
        if (c < 0 || c >= V) l = -INFINITY;
        const bool valid = !(l == -INFINITY);
        any |= valid;
        nan |= valid && !(l == l);
        top = fmaxf(top, l);
        key[j] = ((uint64_t)(valid ? (uint32_t)c : 0x7fffffffu) << 32) | (uint32_t)j;
        prob[j] = l;
    }
    top = warp_max(top);
    any = __any_sync(0xffffffffu, any);
    nan = __any_sync(0xffffffffu, nan);
    if (nan) top = 0.0f;                               // the row's result is NaN whatever the reference point
    float sum = 0.0f;
    for (int32_t j = lane; j < Kp; j += 32) sum += prob[j] == -INFINITY ? 0.0f : expf((prob[j] - top) * inv_tau);
    sum = warp_sum(sum);
    const float inv = any ? 1.0f / sum : 0.0f, log_sum = any ? logf(sum) : 0.0f;
    float plogp = 0.0f, total = 0.0f;
    for (int32_t j = lane; j < Kp; j += 32) {
        const float l = prob[j];
        float q = 0.0f;
        if (l != -INFINITY) {
            const float e = (l - top) * inv_tau;       // the difference first: the lowest finite logit stays finite
            q = expf(e) * inv;
            if (!(q == 0.0f)) plogp = fmaf(q, e - log_sum, plogp);
            total += q;
        }
        prob[j] = q;
    }
    plogp = warp_sum(plogp);
    total = warp_sum(total);
    __syncwarp();
    // bitonic sort of Kp keys
    for (int32_t size = 2; size <= Kp; size <<= 1) {
        for (int32_t d = size >> 1; d > 0; d >>= 1) {
            for (int32_t n = lane; n < (Kp >> 1); n += 32) {
                const int32_t i = 2 * n - (n & (d - 1)), j = i + d;
                const uint64_t a = key[i], b = key[j];
                const bool up = (i & size) == 0;
                if ((a > b) == up) { key[i] = b; key[j] = a; }
            }
            __syncwarp();
        }
    }
    for (int32_t j = lane; j < K; j += 32) {
        const uint64_t k = key[j];
        list[t * K + j] = make_int2((int32_t)(k >> 32), __float_as_int(prob[(uint32_t)k]));
    }
    // where each unit of classes begins: entry j is the first one of the units behind entry j - 1's up to its own.  Put
    // together in shared memory: stores of two bytes all over the row would keep the load / store unit busy for longer than
    // everything else here.
    for (int32_t j = lane; j <= K; j += 32) {
        const int32_t from = j == 0 ? 0 : min((int32_t)(key[j - 1] >> 32) / unit, units) + 1;
        const int32_t to = j == K ? units : min((int32_t)(key[j] >> 32) / unit, units);
        for (int32_t u = from; u <= to; ++u) start[u] = (uint16_t)j;
    }
    __syncwarp();
    uint32_t *out = reinterpret_cast<uint32_t *>(list_start + t * pitch);
    for (int32_t i = lane; i < pitch / 2; i += 32) out[i] = reinterpret_cast<const uint32_t *>(start)[i];
    if (lane == 0) {
        flags[t] = any ? 1 : 0;
        stats[t] = make_float2(plogp, total);
    }
}

// The three bf16 parts of a value, each rounded to nearest from what the ones before leave over: 24 bits, down to 2^-133, where
// bf16 ends.  A first part that rounding up would take out of the range is the largest bf16.
__device__ __forceinline__ void split3(float v, uint16_t &hi, uint16_t &mid, uint16_t &lo) {
    constexpr float kLargest = 3.38953139e38f;         // 2^128 - 2^120
    __nv_bfloat16 h = __float2bfloat16_rn(v);
    if (fabsf(v) > kLargest && fabsf(v) < INFINITY) h = __float2bfloat16_rn(copysignf(kLargest, v));
    float r = v - __bfloat162float(h);
    const __nv_bfloat16 m = __float2bfloat16_rn(r);
    r -= __bfloat162float(m);
    hi = __bfloat16_as_ushort(h);
    mid = __bfloat16_as_ushort(m);
    lo = __bfloat16_as_ushort(__float2bfloat16_rn(r));
}

// ---- operands in the form the contractions read ---------------------------------------------------------------
// Rows padded to 16 bytes, fp32 as three bf16 planes.  Activations are always packed: the kept tokens come to the front.
// Block b < row_blocks owns rows [b * per_block, ...).  It counts the kept rows before its own, by reading the labels again, which
// needs no second launch or hand-over between blocks: at most 592 blocks, each half of the T labels of 8 bytes on average, so
// 19 MB of L2 reads at 8192 tokens, 78 MB at 32768, 2.6 GB at 1.1 million.  The whole launch, d = 64: 7, 17 and 590 us, the
// logits of 1000 classes after it 10, 31 and 880 us.  Then it packs its rows in order.  The last row block zeroes the rows up
// to the next multiple of 64, which the weight gradient contracts over.  The blocks behind pack weights, where they cannot be
// read in place (fp32, or rows that are not a multiple of 16 bytes): all of them, or in the backward one piece of the vocabulary
// (the later pieces without row blocks), so that the workspace does not grow with the vocabulary.
struct PackArgs {
    Labels labels;
    int64_t T, Tpad, per_block;
    int32_t w_rows, d, ld;
    int64_t w_plane_rows;
    unsigned int row_blocks;
    uint16_t *xc, *wc;
    RowInfo *rows;
    int32_t *n_live;
    const float *lse, *dloss;              // backward
    float *loss_out, *lse_out;             // forward: zeroed for the tokens left out
    void *dx;                              // backward: rows zeroed for the tokens left out (or null)
    int dx_bytes;
};

// eight elements of a row from column c, zeros from column d on; dst: their place in the first plane
template <typename TS>
__device__ __forceinline__ void pack8(const TS *__restrict__ src, int32_t c, int32_t d, uint16_t *dst, int64_t plane) {
    alignas(16) uint16_t hi[8], mid[8], lo[8];
    if (sizeof(TS) == 2 && d % 8 == 0 && c + 8 <= d) {
        *reinterpret_cast<uint4 *>(hi) = __ldg(reinterpret_cast<const uint4 *>(src + c));
    } else {
        float v[8];
        if (sizeof(TS) == 4 && d % 4 == 0 && c + 8 <= d) {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(src + c)), b = __ldg(reinterpret_cast<const float4 *>(src + c) + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = c + j < d ? load_as_float(src, c + j) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (sizeof(TS) == 4) split3(v[j], hi[j], mid[j], lo[j]);
            else hi[j] = __bfloat16_as_ushort(__float2bfloat16_rn(v[j]));
        }
    }
    *reinterpret_cast<uint4 *>(dst) = *reinterpret_cast<const uint4 *>(hi);
    if (sizeof(TS) == 4) {
        *reinterpret_cast<uint4 *>(dst + plane) = *reinterpret_cast<const uint4 *>(mid);
        *reinterpret_cast<uint4 *>(dst + 2 * plane) = *reinterpret_cast<const uint4 *>(lo);
    }
}

// A whole row by a warp, lane = column: for rows that are not a multiple of 16 bytes.
template <typename TS>
__device__ __forceinline__ void pack_row(const TS *__restrict__ src, int32_t d, int32_t ld, int lane, uint16_t *dst, int64_t plane) {
    for (int32_t c0 = lane; c0 < ld; c0 += 256) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c0 + 32 * j < d ? load_as_float(src, c0 + 32 * j) : 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int32_t c = c0 + 32 * j;
            if (c >= ld) break;
            if (sizeof(TS) == 4) split3(v[j], dst[c], dst[plane + c], dst[2 * plane + c]);
            else dst[c] = __bfloat16_as_ushort(__float2bfloat16_rn(v[j]));
        }
    }
}

template <typename TS>
__global__ void __launch_bounds__(256)
pack_kernel(const TS *__restrict__ x, const TS *__restrict__ w, const PackArgs a)
{
    __shared__ int warp_count[8];
    __shared__ int32_t slot[256];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_launch_dependents();
    pdl_wait();
    constexpr int kVec = 16 / sizeof(TS);              // rows in whole 16-byte pieces
    const int64_t r0 = (int64_t)blockIdx.x * a.per_block, r1 = min(a.T, r0 + a.per_block);       // r0 < T for every row block
    const int64_t vecs = a.ld >> 3;
    if (blockIdx.x >= a.row_blocks) {                  // weights
        const int64_t plane = a.w_plane_rows * a.ld, block = blockIdx.x - a.row_blocks, blocks = gridDim.x - a.row_blocks;
        if (a.d % kVec != 0) {
            for (int64_t r = block * 8 + warp; r < a.w_rows; r += blocks * 8) pack_row(w + r * a.d, a.d, a.ld, lane, a.wc + r * a.ld, plane);
            return;
        }
        for (int64_t i = block * 256 + threadIdx.x; i < a.w_rows * vecs; i += blocks * 256) {
            const int64_t r = i / vecs;
            const int32_t c = (int32_t)(i - r * vecs) * 8;
            pack8(w + r * a.d, c, a.d, a.wc + r * a.ld + c, plane);
        }
        return;
    }
    int mine = 0;
#pragma unroll 8
    for (int64_t t = threadIdx.x; t < r0; t += 256) mine += a.labels.live(t) ? 1 : 0;
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) warp_count[warp] = mine;
    __syncthreads();
    int64_t base = 0;
    for (int i = 0; i < 8; ++i) base += warp_count[i];

    const int64_t plane = a.Tpad * a.ld;
    for (int64_t b0 = r0; b0 < r1; b0 += 256) {
        const int64_t t = b0 + threadIdx.x;
        const bool live = t < r1 && a.labels.live(t);
        const unsigned int ballot = __ballot_sync(0xffffffffu, live);
        __syncthreads();                               // everyone is done with warp_count and slot
        if (lane == 0) warp_count[warp] = __popc(ballot);
        __syncthreads();
        int64_t at = base + __popc(ballot & ((1u << lane) - 1u));
        for (int i = 0; i < warp; ++i) at += warp_count[i];
        slot[threadIdx.x] = live ? (int32_t)at : -1;
        if (live) {
            RowInfo info;
            info.lse2 = a.lse ? a.lse[t] * kLog2e : 0.0f;
            info.g = a.dloss ? a.dloss[t] : 0.0f;
            info.label = a.labels.flags ? -1 : (int32_t)a.labels.target[t];
            info.row = (int32_t)t;
            a.rows[at] = info;
        } else if (t < r1 && a.loss_out) {
            a.loss_out[t] = 0.0f;
            a.lse_out[t] = 0.0f;
        }
        for (int i = 0; i < 8; ++i) base += warp_count[i];
        __syncthreads();
        const int count = (int)min((int64_t)256, r1 - b0);
        for (int i = warp; i < count; i += 8) {
            const int32_t to = slot[i];
            const int64_t from = b0 + i;
            if (to < 0) {
                if (a.dx) {
                    uint8_t *row = static_cast<uint8_t *>(a.dx) + from * a.d * a.dx_bytes;
                    const int64_t bytes = (int64_t)a.d * a.dx_bytes;
                    if (a.d % 8 == 0) for (int64_t c = lane * 16; c < bytes; c += 512) *reinterpret_cast<uint4 *>(row + c) = make_uint4(0u, 0u, 0u, 0u);
                    else for (int64_t c = lane * 2; c < bytes; c += 64) *reinterpret_cast<uint16_t *>(row + c) = 0;
                }
                continue;
            }
            uint16_t *dst = a.xc + (int64_t)to * a.ld;
            const TS *src = x + from * a.d;
            if (a.d % kVec != 0) {
                pack_row(src, a.d, a.ld, lane, dst, plane);
                continue;
            }
            int32_t c = lane * 8;
            if (sizeof(TS) == 2) {     // four pieces in flight
                for (; c + 3 * 256 + 8 <= a.d; c += 1024) {
                    uint4 v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = __ldg(reinterpret_cast<const uint4 *>(src + c + k * 256));
#pragma unroll
                    for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4 *>(dst + c + k * 256) = v[k];
                }
            }
            for (; c < a.ld; c += 256) pack8(src, c, a.d, dst + c, plane);
        }
    }
    if (blockIdx.x == a.row_blocks - 1) {
        if (threadIdx.x == 0) *a.n_live = (int32_t)base;
        const int64_t end = (base + 63) / 64 * 64;
        for (int64_t i = threadIdx.x; i < (end - base) * vecs; i += 256) {
            uint4 *p = reinterpret_cast<uint4 *>(a.xc + base * a.ld) + i;
#pragma unroll
            for (int pl = 0; pl < (sizeof(TS) == 4 ? 3 : 1); ++pl) p[pl * (plane >> 3)] = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

// ---- forward: join the pieces of a row ------------------------------------------------------------------------
// One warp per token, or a whole block where there are few: every lane merges every 32nd (256th) part, then the lanes (and
// the warps) are merged pairwise, in a fixed order.
struct Joined { float m, s, dot; };
__device__ __forceinline__ void merge(Joined &a, float m, float s, float dot) {
    const float top = fmaxf(a.m, m), ref = top == -INFINITY ? 0.0f : top;
    a.s = a.s * exp2f(a.m - ref) + s * exp2f(m - ref);
    a.m = top;
    a.dot += dot;
}
template <int ROWS>
__global__ void __launch_bounds__(256)
combine_kernel(const float4 *__restrict__ part, int32_t parts, const int32_t *__restrict__ n_live, const RowInfo *__restrict__ rows,
               Labels labels, int32_t n_rows, const float2 *__restrict__ teacher, float tau, float *__restrict__ loss, float *__restrict__ lse)
{
    static_assert(ROWS == 1 || ROWS == 8, "a block or a warp per token");
    constexpr int kLanes = 256 / ROWS;
    __shared__ Joined warps[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = threadIdx.x % kLanes;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t row = (int64_t)blockIdx.x * ROWS + (ROWS == 8 ? warp : 0);
    bool live = row < (n_live ? *n_live : n_rows);
    if (live && !rows && !labels.live(row)) {          // rows in their own order: the ones left out are still among them
        live = false;
        if (sub == 0) { loss[row] = 0.0f; lse[row] = 0.0f; }
    }
    Joined j = {-INFINITY, 0.0f, 0.0f};
    if (live) {
        const float4 *p = part + row * parts;
        int32_t i = sub;
        for (; i + 3 * kLanes < parts; i += 4 * kLanes) {
            const float4 a = p[i], b = p[i + kLanes], c = p[i + 2 * kLanes], d = p[i + 3 * kLanes];
            merge(j, a.x, a.y, a.z); merge(j, b.x, b.y, b.z); merge(j, c.x, c.y, c.z); merge(j, d.x, d.y, d.z);
        }
        for (; i < parts; i += kLanes) { const float4 a = p[i]; merge(j, a.x, a.y, a.z); }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float m = __shfl_down_sync(0xffffffffu, j.m, o), s = __shfl_down_sync(0xffffffffu, j.s, o), d = __shfl_down_sync(0xffffffffu, j.dot, o);
        merge(j, m, s, d);
    }
    if (ROWS == 1) {
        if (lane == 0) warps[warp] = j;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < 8; ++w) merge(j, warps[w].m, warps[w].s, warps[w].dot);
        }
    }
    if (sub == 0 && live) {
        const float lse2 = j.m + log2f(j.s);           // all classes at -infinity: -infinity + log2(0)
        const int64_t t = rows ? (int64_t)rows[row].row : row;
        lse[t] = lse2 * kLn2;
        if (teacher) {
            const float2 e = teacher[t];               // sum p log p, sum p
            loss[t] = tau * (tau * fmaf(kLn2, fmaf(lse2, e.y, -j.dot), e.x));      // tau * tau may be below fp32 where this is not
        } else {
            loss[t] = (lse2 - j.dot) * kLn2;
        }
    }
}

// ---- backward: sums over partial results, one launch per piece where there are any -----------------------------------
struct FinishArgs {
    const int32_t *n_live;
    const RowInfo *rows;
    float tau;
    int32_t planes;
    // db[v0 + c] = sum over the 32-row groups of the kept tokens (bias_blocks blocks of 32 classes)
    const float *col_part;
    int32_t ldz, width;
    float *db;
    unsigned int bias_blocks, dw_blocks, dx_blocks;
    // rows of dw and dx: the sums of their splits
    const float *dw_slots, *dx_slots;
    int32_t dw_splits, dx_splits, d, ld, dw_bf16, dx_bf16;
    int64_t dw_slot_rows, dx_slot_rows;
    void *dw, *dx;                         // dw: the piece's first row
};
// The sums of the splits' rows, times scale, four columns per thread.  Flat over all of them: the rows are few, and a warp per row has too
// few loads in flight (13 us where this takes 5).
__device__ __forceinline__ void join_splits(const float *slots, int32_t splits, int64_t slot_rows, int32_t d, int32_t ld, int64_t n,
                                            const RowInfo *rows, float scale, void *out, int bf16, int64_t first, int64_t stride) {
    const int64_t per_row = (d + 3) / 4, total = n * per_row, split_stride = slot_rows * ld;
    for (int64_t i = first; i < total; i += stride) {
        const int64_t r = total <= 0x7fffffff ? (int64_t)((uint32_t)i / (uint32_t)per_row) : i / per_row;
        const int32_t c = (int32_t)(i - r * per_row) * 4;
        const float *src = slots + r * ld + c;         // a slot's rows are padded: whole pieces of four
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int k = 0; k < splits; ++k) {
            const float4 v = *reinterpret_cast<const float4 *>(src + k * split_stride);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        s.x *= scale; s.y *= scale; s.z *= scale; s.w *= scale;
        const int64_t at = (rows ? (int64_t)rows[r].row : r) * d + c;
        if (d % 4 == 0) {
            if (bf16) {
                const __nv_bfloat162 lo = __floats2bfloat162_rn(s.x, s.y), hi = __floats2bfloat162_rn(s.z, s.w);
                *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(out) + at) =
                    make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
            } else {
                *reinterpret_cast<float4 *>(static_cast<float *>(out) + at) = s;
            }
        } else {
            const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (c + j >= d) break;
                if (bf16) static_cast<__nv_bfloat16 *>(out)[at + j] = __float2bfloat16_rn(v[j]);
                else static_cast<float *>(out)[at + j] = v[j];
            }
        }
    }
}
__global__ void __launch_bounds__(256)
finish_kernel(const FinishArgs a)
{
    __shared__ float sum[8][33];
    pdl_launch_dependents();
    pdl_wait();
    unsigned int b = blockIdx.x;
    const float scale = a.tau * (a.planes == 1 ? common_mantissa(a.rows, *a.n_live) : 1.0f);
    if (b < a.bias_blocks) {
        const int lane = threadIdx.x & 31, g = threadIdx.x >> 5;
        const int32_t groups = (*a.n_live + 31) / 32, c = b * 32 + lane;
        float s = 0.0f;
#pragma unroll 4
        for (int32_t i = g; i < groups; i += 8) s += a.col_part[(int64_t)i * a.ldz + c];
        sum[g][lane] = s;
        __syncthreads();
        if (g == 0 && c < a.width) {
            for (int i = 1; i < 8; ++i) s += sum[i][lane];
            a.db[c] = s * scale;
        }
        return;
    }
    b -= a.bias_blocks;
    if (b < a.dw_blocks) {
        join_splits(a.dw_slots, a.dw_splits, a.dw_slot_rows, a.d, a.ld, a.width, nullptr, scale, a.dw, a.dw_bf16, (int64_t)b * 256 + threadIdx.x,
                    (int64_t)a.dw_blocks * 256);
        return;
    }
    b -= a.dw_blocks;
    join_splits(a.dx_slots, a.dx_splits, a.dx_slot_rows, a.d, a.ld, *a.n_live, a.rows, scale, a.dx, a.dx_bf16, (int64_t)b * 256 + threadIdx.x,
                (int64_t)a.dx_blocks * 256);
}

// ---- workspace ----------------------------------------------------------------------------------------------------
inline size_t pad256(size_t v) { return (v + 255) / 256 * 256; }

struct Plan {
    int planes, pack_w;
    int32_t cols;                          // widest tile: 256 classes or columns, 128 with three planes
    int32_t unit, units, pitch;            // classes per entry of list_start: an epilogue warp's, more where that is a large table
    int32_t ld, bn, parts, width, pieces, dx_splits, dw_splits;
    int32_t w_rows;                        // weights packed at a time
    bool direct;
    int64_t Tpad;
    bool dx_slots, dw_slots;
    size_t o_live, o_rows, o_x, o_w, o_list, o_start, o_flags, o_teacher, o_part, o_dz, o_col, o_dx, o_dw, total;
};

// Classes per tile of a logits launch: the width whose whole rounds over the SM pairs cost least.  A round costs what it
// stages per 64-element step (the token rows that exist and the classes) plus about 64 rows' worth for its hand-over.  The
// widest when there are many rounds, where narrow tiles would only read x more often.
int32_t classes_per_tile(int64_t T, int64_t V, int32_t most, int32_t least, int32_t step)
{
    const int64_t pairs = sm_count() > 1 ? sm_count() / 2 : 74, mt = (T + kTile - 1) / kTile;
    int32_t best = most;
    if (mt * ((V + most - 1) / most) >= 8 * pairs) return best;
    int64_t cost = INT64_MAX;
    for (int32_t bn = most; bn >= least; bn -= step) {
        const int64_t c = (mt * ((V + bn - 1) / bn) + pairs - 1) / pairs * ((T < kTile ? T : kTile) + bn + 64);
        if (c < cost) { cost = c; best = bn; }
    }
    return best;
}

// Time of a gradient launch in units of one 64-element step, for n0 tiles of k0 steps and n1 tiles of k1 steps over the SM
// pairs, longest first (the order of the kernel); `own`: what a tile costs beside its steps.
int64_t grads_makespan(int64_t n0, int64_t k0, int64_t n1, int64_t k1, int64_t own, int64_t pairs)
{
    if (n0 > 0 && (n1 == 0 || k0 >= k1)) { const int64_t n = n0, k = k0; n0 = n1; k0 = k1; n1 = n; k1 = k; }      // 1: the longer
    const int64_t l = k1 + own, sh = k0 + own, a = n1 / pairs, r = n1 % pairs;
    if (r == 0) return a * l + (n0 + pairs - 1) / pairs * sh;
    // r pairs finish their longer tiles at (a + 1) l, the others at a l.  The answer is one of the times at which a pair of one
    // kind or the other finishes a shorter tile, whichever comes first with room for all of them.
    const int64_t first = l / sh, started = (l + sh - 1) / sh;        // shorter tiles of a pair that is early, done and begun by (a + 1) l
    const int64_t rest = n0 - (pairs - r) * first, late = rest > 0 ? (rest + pairs - 1) / pairs : 0;
    const int64_t need = (n0 + r * started + pairs - 1) / pairs, early = need > started ? need : started;
    const int64_t t_late = (a + 1) * l + late * sh, t_early = a * l + early * sh;
    return t_late < t_early ? t_late : t_early;
}

// Tile counts follow from the sizes alone; how many tokens are kept is known on the device only.
Plan make_plan(int64_t T, int32_t d, int32_t V, int dtype, int32_t K, bool backward)
{
    Plan p = {};
    p.planes = dtype == TBN_F32 ? 3 : 1;
    p.cols = dtype == TBN_F32 ? 128 : 256;
    constexpr int32_t groups = 2;                      // epilogue warps that share a tile's columns
    p.ld = (d + 63) / 64 * 64;                         // packed rows are whole 64-column panels
    p.pack_w = dtype == TBN_F32 || d % 8 != 0;
    p.Tpad = round_up64(T, kTile);
    const int64_t Vpad = round_up64(V, kTile);
    // One tile of tokens in bf16: the forward reads x in place and leaves the dropped rows' results out at the end; with
    // more tokens, dropping them first pays for its launch.
    p.direct = !backward && T <= kTile && !p.pack_w;
    size_t o = 0;
    auto take = [&o](size_t bytes) { const size_t at = o; o += pad256(bytes); return at; };
    p.o_live = take(4);
    p.o_rows = take(p.direct ? 0 : (size_t)p.Tpad * sizeof(RowInfo));
    p.o_x = take(p.direct ? 0 : (size_t)p.planes * p.Tpad * p.ld * 2);
    p.o_list = take((size_t)T * K * 8);
    p.o_flags = take(K > 0 ? (size_t)T : 0);
    p.o_teacher = take(K > 0 ? (size_t)T * 8 : 0);
    if (!backward) {
        p.bn = classes_per_tile(T, V, p.cols, 64, 32);
        p.parts = (int32_t)((V + p.bn - 1) / p.bn * groups);
        p.o_part = take((size_t)p.parts * p.Tpad * sizeof(float4));
    } else {
        int64_t width = (int64_t)(kPieceBytes / ((size_t)2 * p.planes * p.Tpad)) / kTile * kTile;
        if (width < 1024) width = 1024;
        if (width > Vpad) width = Vpad;
        p.pieces = (int32_t)((Vpad + width - 1) / width);
        p.width = (int32_t)round_up64((Vpad + p.pieces - 1) / p.pieces, kTile);
        p.pieces = (int32_t)((Vpad + p.width - 1) / p.width);
        p.bn = classes_per_tile(T, V < p.width ? V : p.width, p.cols, 128, 64);       // whole chunks of 32 classes per warp
        // A contraction is split when its few tiles would outlast the rest of the launch.  A split adds its share of the
        // fp32 partial sums, written here and read by the pass that joins them: 8 bytes per element and split at a few
        // TB/s, about 1 step per 2 M elements.  A tile costs about 10 steps beside its products (64 x 512 x 30000, whole
        // gradient: counted as 6 steps, 14 splits and 68 us; as 12, 9 splits and 59 us).  A step of the six-product form takes
        // three times as long.
        const int64_t nt = (d + p.cols - 1) / p.cols, mt = p.Tpad / kTile, vt = (V < p.width ? round_up64(V, kTile) : p.width) / kTile;
        const int64_t kx = p.width / 64, kw = (T + 63) / 64, pairs = sm_count() > 1 ? sm_count() / 2 : 74;
        const int64_t own = p.planes == 1 ? 10 : 3, per_step = (p.planes == 1 ? 2 : 6) << 20;
        int64_t best = INT64_MAX;
        p.dx_splits = p.dw_splits = 1;
        for (int32_t i = 1; i <= kMaxSplits && (i == 1 || 2 * i <= kx); ++i) {
            for (int32_t j = 1; j <= kMaxSplits && (j == 1 || 2 * j <= kw); ++j) {
                if (j > 1 && vt * nt * j > 4 * pairs) break;
                const int64_t join = (i > 1 ? i * p.Tpad * d : 0) + (j > 1 ? j * vt * kTile * d : 0);
                const int64_t c = grads_makespan(mt * nt * i, (kx + i - 1) / i, vt * nt * j, (kw + j - 1) / j, own, pairs) + join / per_step +
                                  (join > 0 ? own : 0);
                if (c < best) { best = c; p.dx_splits = i; p.dw_splits = j; }
            }
            if (mt * nt * i > 4 * pairs) break;
        }
        p.dx_slots = p.dx_splits > 1 || (p.pieces > 1 && dtype == TBN_BF16);
        p.dw_slots = p.dw_splits > 1;
        p.o_dz = take((size_t)p.planes * p.Tpad * p.width * 2);
        p.o_col = take((size_t)(p.Tpad / 32) * p.width * 4);
        p.o_dx = take(p.dx_slots ? (size_t)p.dx_splits * p.Tpad * p.ld * 4 : 0);
        p.o_dw = take(p.dw_slots ? (size_t)p.dw_splits * p.width * p.ld * 4 : 0);
    }
    p.w_rows = backward && p.width < V ? p.width : V;
    p.o_w = take(p.pack_w ? (size_t)p.planes * p.w_rows * p.ld * 2 : 0);
    if (K > 0) {
        p.unit = p.bn / groups;
        while (V / p.unit >= kMaxUnits || (T * (V / p.unit) > ((int64_t)1 << 26) && V / p.unit > 1)) p.unit *= 2;
        p.units = (int32_t)(((int64_t)V + p.unit - 1) / p.unit);
        p.pitch = (p.units + 2) / 2 * 2;               // units + 1 entries in whole 32-bit words
        p.o_start = take((size_t)T * p.pitch * 2);
    }
    p.total = o;
    return p;
}

// The first kernel of a call that has the GPU's every SM to fill, launched the ordinary way.  Launched early (launch_pdl), its
// blocks are placed while the kernel before it still holds most SMs with its shared memory, all on the few that are free, and
// stay there: the teacher's lists of 512 tokens took 26 us that way and take 9.6, those of 2048 tokens 25 and 10.8.  The packing
// kernel after it is better off early (6.7 and 4.9 us).
template <typename... KArgs, typename... Args>
cudaError_t launch_spread(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = s;
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

unsigned blocks_for(int64_t items, int64_t per_block, int64_t most)
{
    int64_t b = (items + per_block - 1) / per_block;
    return (unsigned)(b < 1 ? 1 : b > most ? most : b);
}

// The packing launch: the rows that `a` asks for, and the weights of the piece that begins at class v0.
cudaError_t pack(const HeadCall &c, const Plan &p, char *ws, PackArgs a, int32_t v0, cudaStream_t s)
{
    a.w_rows = c.V - v0 < p.w_rows ? c.V - v0 : p.w_rows;
    a.w_plane_rows = p.w_rows; a.d = c.d; a.ld = p.ld;
    a.wc = reinterpret_cast<uint16_t *>(ws + p.o_w);
    const unsigned blocks = a.row_blocks + (p.pack_w ? blocks_for((int64_t)a.w_rows * (p.ld / 8), 256, 2368) : 0u);
    const int64_t w0 = (int64_t)v0 * c.d;
    return c.dtype == TBN_F32 ? launch_pdl(pack_kernel<float>, dim3(blocks), dim3(256), 0, s, static_cast<const float *>(c.x),
                                           static_cast<const float *>(c.w) + w0, a)
                              : launch_pdl(pack_kernel<__nv_bfloat16>, dim3(blocks), dim3(256), 0, s,
                                           static_cast<const __nv_bfloat16 *>(c.x), static_cast<const __nv_bfloat16 *>(c.w) + w0, a);
}

// Labels, operands and per-row values: everything before the first contraction.
int prepare(const HeadCall &c, const Plan &p, char *ws, bool backward, LogitsArgs *out, cudaStream_t s)
{
    out->status = device_status_ptr();
    if (!out->status) return TBN_ERR_CUDA;
    int32_t *n_live = reinterpret_cast<int32_t *>(ws + p.o_live);
    RowInfo *rows = reinterpret_cast<RowInfo *>(ws + p.o_rows);
    Labels labels = {c.targets, c.ignore_index, c.V, nullptr};

    if (c.K > 0) {
        int32_t Kp = 32;
        while (Kp < c.K) Kp <<= 1;
        const int warps = teacher_warps(Kp);
        const size_t smem = teacher_smem(Kp, p.pitch) * warps;
        const dim3 grid((unsigned)((c.T + warps - 1) / warps));
        int2 *list = reinterpret_cast<int2 *>(ws + p.o_list);
        uint8_t *flags = reinterpret_cast<uint8_t *>(ws + p.o_flags);
        float2 *stats = reinterpret_cast<float2 *>(ws + p.o_teacher);
        uint16_t *start = reinterpret_cast<uint16_t *>(ws + p.o_start);
        const cudaError_t e = c.top_dtype == TBN_F32
            ? launch_spread(teacher_kernel<float>, grid, dim3(32 * warps), smem, s, c.top_index, static_cast<const float *>(c.top_logit),
                         c.T, c.K, Kp, c.V, 1.0f / c.tau, p.unit, p.units, p.pitch, list, start, flags, stats)
            : launch_spread(teacher_kernel<__nv_bfloat16>, grid, dim3(32 * warps), smem, s, c.top_index,
                         static_cast<const __nv_bfloat16 *>(c.top_logit), c.T, c.K, Kp, c.V, 1.0f / c.tau, p.unit, p.units,
                         p.pitch, list, start, flags, stats);
        if (e != cudaSuccess) return TBN_ERR_CUDA;
        labels.flags = flags;
        labels.target = nullptr;
        out->list = list;
        out->list_start = start;
        out->K = c.K;
        out->unit = p.unit;
        out->units = p.units;
        out->pitch = p.pitch;
    }
    out->labels = labels;
    const int32_t w_ld = p.pack_w ? p.ld : c.d;
    out->w = Operand{p.pack_w ? static_cast<const void *>(ws + p.o_w) : c.w, p.pack_w ? p.w_rows : c.V, p.pack_w ? p.w_rows : c.V, w_ld, w_ld};
    out->planes = p.planes; out->bn = p.bn;
    out->bias = c.bias; out->scale2 = kLog2e / c.tau; out->T = c.T; out->Tpad = p.Tpad;
    if (p.direct) {
        out->x = Operand{c.x, c.T, c.T, c.d, c.d};
        return TBN_OK;
    }
    PackArgs a = {};
    a.labels = labels; a.T = c.T; a.Tpad = p.Tpad;
    a.per_block = (c.T + 591) / 592 < 8 ? 8 : (c.T + 591) / 592;
    a.row_blocks = (unsigned)((c.T + a.per_block - 1) / a.per_block);              // the last one has rows of its own
    a.xc = reinterpret_cast<uint16_t *>(ws + p.o_x);
    a.rows = rows; a.n_live = n_live;
    if (backward) {
        a.lse = c.lse; a.dloss = c.dloss; a.dx = c.dx; a.dx_bytes = c.dx_dtype == TBN_F32 ? 4 : 2;
    } else {
        a.loss_out = c.loss_out; a.lse_out = c.lse_out;
    }
    if (pack(c, p, ws, a, 0, s) != cudaSuccess) return TBN_ERR_CUDA;
    out->x = Operand{ws + p.o_x, p.Tpad, p.Tpad, p.ld, p.ld};
    out->n_live = n_live; out->rows = rows;
    return TBN_OK;
}

}  // namespace

size_t workspace_bytes(int64_t T, int32_t d, int32_t V, int dtype, int32_t K, bool backward)
{
    return make_plan(T, d, V, dtype, K, backward).total;
}

int forward(const HeadCall &c, void *workspace, size_t workspace_bytes, cudaStream_t s)
{
    const Plan p = make_plan(c.T, c.d, c.V, c.dtype, c.K, false);
    if (!workspace || workspace_bytes < p.total) return TBN_ERR_WORKSPACE;
    char *ws = static_cast<char *>(workspace);
    LogitsArgs a = {};
    int rc = prepare(c, p, ws, false, &a, s);
    if (rc != TBN_OK) return rc;
    a.v0 = 0; a.width = c.V;
    a.part = reinterpret_cast<float4 *>(ws + p.o_part);
    a.parts = p.parts;
    rc = launch_head_stats(a, s);
    if (rc != TBN_OK) return rc;
    const float2 *teacher = c.K > 0 ? reinterpret_cast<const float2 *>(ws + p.o_teacher) : nullptr;
    // enough blocks for the GPU: one row per block when there are few tokens
    const int rb = c.T >= 256 ? 8 : 1;
    const dim3 grid((unsigned)((c.T + rb - 1) / rb));
    auto kern = rb == 8 ? combine_kernel<8> : combine_kernel<1>;
    return launch_pdl(kern, grid, dim3(256), 0, s, static_cast<const float4 *>(a.part), p.parts, a.n_live, a.rows, a.labels,
                      (int32_t)c.T, teacher, c.tau, c.loss_out, c.lse_out) == cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
}

int backward(const HeadCall &c, void *workspace, size_t workspace_bytes, cudaStream_t s)
{
    const bool dx_bf16 = c.dx_dtype == TBN_BF16;       // dx has the operands' type
    const Plan p = make_plan(c.T, c.d, c.V, c.dtype, c.K, true);
    if (!workspace || workspace_bytes < p.total) return TBN_ERR_WORKSPACE;
    char *ws = static_cast<char *>(workspace);
    LogitsArgs a = {};
    int rc = prepare(c, p, ws, true, &a, s);
    if (rc != TBN_OK) return rc;
    a.dz = ws + p.o_dz;
    a.ldz = p.width;
    a.col_part = c.db ? reinterpret_cast<float *>(ws + p.o_col) : nullptr;

    GradArgs g = {};
    g.x = a.x; g.w = a.w; g.planes = a.planes; g.n_live = a.n_live; g.rows = a.rows; g.tau = c.tau; g.dz = a.dz;
    g.T = c.T; g.Tpad = p.Tpad; g.d = c.d; g.ldz = p.width;
    g.want_dx = c.dx != nullptr; g.want_dw = c.dw != nullptr;
    g.dx = c.dx; g.dx_bf16 = dx_bf16; g.dx_slots = p.dx_slots ? reinterpret_cast<float *>(ws + p.o_dx) : nullptr; g.dx_splits = p.dx_splits;
    g.dw = c.dw; g.dw_bf16 = c.dw_dtype == TBN_BF16; g.dw_slots = p.dw_slots ? reinterpret_cast<float *>(ws + p.o_dw) : nullptr;
    g.dw_splits = p.dw_splits;
    g.slot_ld = p.ld;
    g.status = a.status;
    for (int32_t piece = 0; piece < p.pieces; ++piece) {
        a.v0 = piece * p.width;
        a.width = c.V - a.v0 < p.width ? c.V - a.v0 : p.width;
        a.w_row0 = g.w_row0 = p.pack_w ? 0 : a.v0;
        if (p.pack_w) a.w.rows = g.w.rows = a.width;
        if (p.pack_w && piece > 0 && pack(c, p, ws, PackArgs{}, a.v0, s) != cudaSuccess) return TBN_ERR_CUDA;
        rc = launch_head_dz(a, s);
        if (rc != TBN_OK) return rc;
        const bool grads = g.want_dx || g.want_dw, last = piece == p.pieces - 1;
        if (grads) {
            g.v0 = a.v0; g.width = a.width;
            g.dx_add = piece > 0;
            g.dx_last = last;
            rc = launch_head_grads(g, s);
            if (rc != TBN_OK) return rc;
        }
        FinishArgs f = {};
        f.n_live = a.n_live; f.rows = a.rows; f.tau = c.tau; f.planes = p.planes; f.d = c.d; f.ld = p.ld; f.width = a.width;
        if (c.db) {
            f.col_part = a.col_part; f.ldz = a.ldz; f.db = c.db + a.v0;
            f.bias_blocks = (unsigned)((a.width + 31) / 32);
        }
        if (g.want_dw && p.dw_splits > 1) {
            f.dw_blocks = blocks_for((int64_t)a.width * c.d, 1024, 1184);
            f.dw_slots = g.dw_slots; f.dw_splits = p.dw_splits; f.dw_slot_rows = round_up64(a.width, kTile); f.dw_bf16 = g.dw_bf16;
            f.dw = static_cast<char *>(c.dw) + (int64_t)a.v0 * c.d * (g.dw_bf16 ? 2 : 4);
        }
        if (g.want_dx && p.dx_splits > 1 && last) {
            f.dx_blocks = blocks_for(c.T * c.d, 1024, 1184);
            f.dx_slots = g.dx_slots; f.dx_splits = p.dx_splits; f.dx_slot_rows = p.Tpad; f.dx_bf16 = dx_bf16; f.dx = c.dx;
        }
        const unsigned blocks = f.bias_blocks + f.dw_blocks + f.dx_blocks;
        if (blocks && launch_pdl(finish_kernel, dim3(blocks), dim3(256), 0, s, f) != cudaSuccess) return TBN_ERR_CUDA;
    }
    return TBN_OK;
}

}  // namespace head
}  // namespace tbn
