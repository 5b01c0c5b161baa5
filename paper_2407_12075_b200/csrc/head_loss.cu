// Losses of a large-vocabulary head: labels, operand packing, reductions and the order of the launches.  The
// contractions are in tc_head.cu.
//
//   z_tv = x_t . w_v + b_v;  lse_t = log sum_v exp(z_tv / tau)
//   cross entropy (tau = 1)   loss_t = lse_t - z_t,label
//   distillation              loss_t = tau^2 sum_j p_tj (log p_tj - z_t,idx(t,j) / tau + lse_t)
//   gradient                  dz_tv = dloss_t tau (exp(z_tv / tau - lse_t) - sum_{j: idx(t,j) = v} p_tj)
//
// Cross entropy is distillation from one entry of probability 1, so both share every kernel; only where the entries come
// from differs.  The logits are never stored: the forward keeps one (maximum, sum, weighted dot) triple per token and 128
// classes, the backward recomputes the logits piece by piece of the vocabulary and stores dz for one piece at a time.
//
// Tokens that are left out (ignored targets, empty teacher rows) are dropped first: the kept rows are packed to the front,
// so no kernel computes anything for the others and nothing in their rows -- infinities, NaN -- can reach a result.
#include <cuda_fp16.h>

#include <climits>

#include "head_loss.cuh"

namespace tbn {
namespace head {

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr size_t kPieceBytes = (size_t)256 << 20;      // bound on one piece of dz (a piece has at least 1024 classes)

// ---- which tokens take part -------------------------------------------------------------------------
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

// ---- the teacher's entries ---------------------------------------------------------------------------
// One warp per token: p = softmax(logit / tau) over the entries whose index is a class and whose logit is above
// -infinity, sum p log p, and the entries sorted by class (by position among equals), which is the order in which the
// epilogues meet the classes.
constexpr int kTeacherWarps = 4;

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

template <typename TL>
__global__ void __launch_bounds__(32 * kTeacherWarps)
teacher_kernel(const int64_t *__restrict__ index, const TL *__restrict__ logit, int64_t T, int32_t K, int32_t Kp, int32_t V,
               float inv_tau, int32_t *__restrict__ list_idx, float *__restrict__ list_p, uint8_t *__restrict__ flags,
               float2 *__restrict__ stats)
{
    extern __shared__ uint8_t teacher_smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint64_t *key = reinterpret_cast<uint64_t *>(teacher_smem) + (size_t)warp * Kp;
    float *prob = reinterpret_cast<float *>(reinterpret_cast<uint64_t *>(teacher_smem) + (size_t)kTeacherWarps * Kp) + (size_t)warp * Kp;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t t = (int64_t)blockIdx.x * kTeacherWarps + warp;
    if (t >= T) return;
    float top = -INFINITY;
    bool any = false, nan = false;
    for (int32_t j = lane; j < Kp; j += 32) {
        int64_t c = -1;
        float l = -INFINITY;
        if (j < K) {
            c = index[t * K + j];
            if (c >= 0 && c < V) l = load_as_float(logit, t * K + j) * inv_tau;
        }
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
    for (int32_t j = lane; j < Kp; j += 32) sum += prob[j] == -INFINITY ? 0.0f : expf(prob[j] - top);
    sum = warp_sum(sum);
    const float inv = any ? 1.0f / sum : 0.0f, log_sum = any ? logf(sum) : 0.0f;
    float plogp = 0.0f, total = 0.0f;
    for (int32_t j = lane; j < Kp; j += 32) {
        const float l = prob[j];
        float q = 0.0f;
        if (l != -INFINITY) {
            q = expf(l - top) * inv;
            if (!(q == 0.0f)) plogp = fmaf(q, l - top - log_sum, plogp);
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
        list_idx[t * K + j] = (int32_t)(k >> 32);
        list_p[t * K + j] = prob[(uint32_t)k];
    }
    if (lane == 0) {
        flags[t] = any ? 1 : 0;
        stats[t] = make_float2(plogp, total);
    }
}

// ---- fp32 operands: largest magnitudes ------------------------------------------------------------------
// max_bits[0..2]: bit patterns of max |x| over the kept rows, max |w|, max |dloss * tau| over the kept rows (a maximum does
// not depend on the order in which it is taken).
__device__ __forceinline__ void fold_max(unsigned int *slot, float v) {
    v = warp_max(v);
    __shared__ float part[8];
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x < 32) {
        v = threadIdx.x < (blockDim.x >> 5) ? part[threadIdx.x] : 0.0f;
        v = warp_max(v);
        if (threadIdx.x == 0 && v > 0.0f) atomicMax(slot, __float_as_uint(v));
    }
}
__global__ void __launch_bounds__(256)
abs_max_kernel(const float *__restrict__ x, Labels labels, int64_t T, int32_t d, const float *__restrict__ w, int64_t w_count,
               const float *__restrict__ dloss, float tau, unsigned int *__restrict__ max_bits)
{
    pdl_launch_dependents();
    pdl_wait();
    const int64_t tid = (int64_t)blockIdx.x * 256 + threadIdx.x, threads = (int64_t)gridDim.x * 256;
    float mw = 0.0f, mx = 0.0f, mg = 0.0f;
    const int64_t w4 = w_count >> 2;
    const float4 *wv = reinterpret_cast<const float4 *>(w);
    for (int64_t i = tid; i < w4; i += threads) {
        const float4 v = __ldg(wv + i);
        mw = fmaxf(mw, fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w))));
    }
    for (int64_t i = (w4 << 2) + tid; i < w_count; i += threads) mw = fmaxf(mw, fabsf(w[i]));
    const int lane = threadIdx.x & 31;
    for (int64_t t = tid >> 5; t < T; t += threads >> 5) {
        if (!labels.live(t)) continue;
        for (int32_t c = lane; c < d; c += 32) mx = fmaxf(mx, fabsf(x[t * d + c]));
        if (dloss && lane == 0) mg = fmaxf(mg, fabsf(dloss[t] * tau));
    }
    __syncwarp();
    fold_max(max_bits + 0, mx);
    fold_max(max_bits + 1, mw);
    fold_max(max_bits + 2, mg);
}
// The power of two that takes the largest magnitude to [2^14, 2^15): the high part of every element then keeps 11 bits
// and the remainder another 11, down to 2^-38 of the largest one, below which fp16 ends.  Non-finite or zero: 1.
__device__ __forceinline__ float scale_of(unsigned int bits) {
    const float m = __uint_as_float(bits);
    if (!(m > 0.0f) || !(m < INFINITY)) return 1.0f;
    int e = (int)(bits >> 23) - 127;                   // subnormal maxima: -127, clamped below
    e = e > 60 ? 60 : e < -60 ? -60 : e;
    return __uint_as_float((unsigned int)(127 + 14 - e) << 23);
}
__device__ __forceinline__ void split16(float v, __half &hi, __half &lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(v - __half2float(hi));
}

// ---- weights in the form the contractions read: padded rows, fp32 as two fp16 planes --------------------------
// Needed for fp32 weights and for rows that are not a multiple of 16 bytes; other weights are read in place.
template <typename TW>
__global__ void __launch_bounds__(256)
pack_weight_kernel(const TW *__restrict__ w, int64_t V, int32_t d, int32_t ld, const unsigned int *__restrict__ max_bits,
                   uint16_t *__restrict__ out)
{
    pdl_launch_dependents();
    pdl_wait();
    const float sc = sizeof(TW) == 4 ? scale_of(max_bits[1]) : 1.0f;
    const int64_t groups = V * (ld >> 3), plane = V * ld;
    const bool vec = sizeof(TW) == 4 && d % 4 == 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < groups; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / (ld >> 3);
        const int32_t c = (int32_t)(i - r * (ld >> 3)) * 8;
        alignas(16) uint16_t hi[8], lo[8];
        float v[8];
        if (vec && c + 8 <= d) {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(w + r * d + c)), b = __ldg(reinterpret_cast<const float4 *>(w + r * d + c + 4));
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = c + j < d ? load_as_float(w, r * d + c + j) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (sizeof(TW) == 4) {
                __half h, l;
                split16(v[j] * sc, h, l);
                hi[j] = __half_as_ushort(h); lo[j] = __half_as_ushort(l);
            } else {
                hi[j] = __bfloat16_as_ushort(__float2bfloat16_rn(v[j]));
            }
        }
        *reinterpret_cast<uint4 *>(out + r * ld + c) = *reinterpret_cast<const uint4 *>(hi);
        if (sizeof(TW) == 4) *reinterpret_cast<uint4 *>(out + plane + r * ld + c) = *reinterpret_cast<const uint4 *>(lo);
    }
}

// ---- kept tokens to the front ---------------------------------------------------------------------------------
// Block b owns rows [b * per_block, ...).  It counts the kept rows before its own (re-reading the labels: at most a few
// hundred blocks, so a few megabytes of L2 reads for tens of thousands of tokens, and no second launch or hand-over
// between blocks), then packs its rows in order.  The last block zeroes the rows up to the next multiple of 64, which the
// weight gradient contracts over.
struct PackArgs {
    Labels labels;
    int64_t T, Tpad, per_block;
    int32_t d, ld;
    const unsigned int *max_bits;          // fp32 only
    uint16_t *xc;
    RowInfo *rows;
    int32_t *n_live;
    Scales *scales;                        // fp32 only: written here for the kernels that follow
    float tau;
    const float *lse, *dloss;              // backward
    float *loss_out, *lse_out;             // forward: zeroed for the tokens left out
    void *dx;                              // backward: rows zeroed for the tokens left out (or null)
    int dx_bytes;
};
template <typename TX>
__global__ void __launch_bounds__(256)
pack_rows_kernel(const TX *__restrict__ x, PackArgs a)
{
    __shared__ int warp_count[8];
    __shared__ int32_t slot[256];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t r0 = min(a.T, (int64_t)blockIdx.x * a.per_block), r1 = min(a.T, r0 + a.per_block);
    int mine = 0;
    for (int64_t t = threadIdx.x; t < r0; t += 256) mine += a.labels.live(t) ? 1 : 0;
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) warp_count[warp] = mine;
    __syncthreads();
    int64_t base = 0;
    for (int i = 0; i < 8; ++i) base += warp_count[i];

    float sx = 1.0f, sg = 1.0f;
    if (sizeof(TX) == 4) {
        sx = scale_of(a.max_bits[0]);
        if (a.dloss) sg = scale_of(a.max_bits[2]);
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            const float sw = scale_of(a.max_bits[1]);
            *a.scales = Scales{sx, sw, sg, 1.0f / sx, 1.0f / sw, 1.0f / sg};
        }
    }
    const int64_t plane = a.Tpad * a.ld;
    const bool vec = a.d % 8 == 0;
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
            info.g = a.dloss ? a.dloss[t] * a.tau * sg : 0.0f;
            info.label = a.labels.target ? (int32_t)a.labels.target[t] : -1;
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
                    if (vec) for (int64_t c = lane * 16; c < bytes; c += 512) *reinterpret_cast<uint4 *>(row + c) = make_uint4(0u, 0u, 0u, 0u);
                    else for (int64_t c = lane * 2; c < bytes; c += 64) *reinterpret_cast<uint16_t *>(row + c) = 0;
                }
                continue;
            }
            const TX *src = x + from * a.d;
            uint16_t *dst = a.xc + (int64_t)to * a.ld;
            for (int32_t c = lane * 8; c < a.ld; c += 256) {
                alignas(16) uint16_t hi[8], lo[8];
                if (sizeof(TX) == 2 && vec) {
                    *reinterpret_cast<uint4 *>(hi) = __ldg(reinterpret_cast<const uint4 *>(src + c));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float v = c + j < a.d ? load_as_float(src, c + j) : 0.0f;
                        if (sizeof(TX) == 4) {
                            __half h, l;
                            split16(v * sx, h, l);
                            hi[j] = __half_as_ushort(h); lo[j] = __half_as_ushort(l);
                        } else {
                            hi[j] = __bfloat16_as_ushort(__float2bfloat16_rn(v));
                        }
                    }
                }
                *reinterpret_cast<uint4 *>(dst + c) = *reinterpret_cast<const uint4 *>(hi);
                if (sizeof(TX) == 4) *reinterpret_cast<uint4 *>(dst + plane + c) = *reinterpret_cast<const uint4 *>(lo);
            }
        }
    }
    if (blockIdx.x == gridDim.x - 1) {
        if (threadIdx.x == 0) *a.n_live = (int32_t)base;
        const int64_t end = (base + 63) / 64 * 64, vecs = (end - base) * (a.ld >> 3);
        for (int64_t i = threadIdx.x; i < vecs; i += 256) {
            uint4 *p = reinterpret_cast<uint4 *>(a.xc + base * a.ld) + i;
            *p = make_uint4(0u, 0u, 0u, 0u);
            if (sizeof(TX) == 4) *(p + (plane >> 3)) = make_uint4(0u, 0u, 0u, 0u);
        }
    }
}

// ---- forward: join the pieces of a row ------------------------------------------------------------------------
// RB rows x (256 / RB) threads: every thread merges every (256 / RB)-th triple, then the threads of a row are merged in a
// fixed order.
template <int RB>
__global__ void __launch_bounds__(256)
combine_kernel(const float *__restrict__ part_max, const float *__restrict__ part_sum, const float *__restrict__ part_dot, int32_t parts,
               int64_t Tpad, const int32_t *__restrict__ n_live, const RowInfo *__restrict__ rows, const float2 *__restrict__ teacher,
               float tau, float *__restrict__ loss, float *__restrict__ lse)
{
    constexpr int kParts = 256 / RB;
    __shared__ float sm[256], ss[256], sd[256];
    const int r = threadIdx.x % RB, g = threadIdx.x / RB;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t row = (int64_t)blockIdx.x * RB + r;
    const bool live = row < *n_live;
    float m = -INFINITY, s = 0.0f, dot = 0.0f;
    if (live) {
#pragma unroll 4
        for (int32_t i = g; i < parts; i += kParts) {
            const int64_t at = (int64_t)i * Tpad + row;
            const float pm = part_max[at], ps = part_sum[at];
            dot += part_dot[at];
            const float mn = fmaxf(m, pm), ref = mn == -INFINITY ? 0.0f : mn;
            s = s * exp2f(m - ref) + ps * exp2f(pm - ref);
            m = mn;
        }
    }
    sm[threadIdx.x] = m; ss[threadIdx.x] = s; sd[threadIdx.x] = dot;
    __syncthreads();
    if (g == 0 && live) {
        for (int i = 1; i < kParts; ++i) {
            const float pm = sm[i * RB + r], ps = ss[i * RB + r];
            dot += sd[i * RB + r];
            const float mn = fmaxf(m, pm), ref = mn == -INFINITY ? 0.0f : mn;
            s = s * exp2f(m - ref) + ps * exp2f(pm - ref);
            m = mn;
        }
        const float lse2 = m + log2f(s);               // all classes at -infinity: -infinity + log2(0)
        const int32_t t = rows[row].row;
        lse[t] = lse2 * kLn2;
        if (teacher) {
            const float2 e = teacher[t];               // sum p log p, sum p
            loss[t] = tau * tau * fmaf(kLn2, fmaf(lse2, e.y, -dot), e.x);
        } else {
            loss[t] = (lse2 - dot) * kLn2;
        }
    }
}

// ---- backward: sums over partial results ------------------------------------------------------------------------
// db[v0 + c] = sum over the 32-row groups of the kept tokens
__global__ void __launch_bounds__(256)
bias_grad_kernel(const float *__restrict__ part, int32_t ld, const int32_t *__restrict__ n_live, const Scales *__restrict__ scales,
                 int32_t width, float *__restrict__ db)
{
    __shared__ float sum[8][33];
    const int lane = threadIdx.x & 31, g = threadIdx.x >> 5;
    pdl_launch_dependents();
    pdl_wait();
    const int32_t groups = (*n_live + 31) / 32;
    const int32_t c = blockIdx.x * 32 + lane;
    float s = 0.0f;
#pragma unroll 4
    for (int32_t i = g; i < groups; i += 8) s += part[(int64_t)i * ld + c];
    sum[g][lane] = s;
    __syncthreads();
    if (g == 0 && c < width) {
        for (int i = 1; i < 8; ++i) s += sum[i][lane];
        db[c] = scales ? s * scales->inv_g : s;
    }
}

// out[row(i)][:] = sum of the splits' partial rows i (rows == nullptr: row(i) = i, `count` rows)
template <typename TO>
__global__ void __launch_bounds__(256)
join_splits_kernel(const float *__restrict__ slots, int32_t splits, int64_t slot_rows, int32_t d, const int32_t *__restrict__ n_live,
                   const RowInfo *__restrict__ rows, int64_t count, TO *__restrict__ out)
{
    pdl_launch_dependents();
    pdl_wait();
    const int64_t n = rows ? *n_live : count;
    const int64_t total = n * d, split_stride = slot_rows * d;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        float s = 0.0f;
        for (int k = 0; k < splits; ++k) s += slots[k * split_stride + i];
        const int64_t r = i / d;
        store_from_float(out, (rows ? (int64_t)rows[r].row : r) * d + (i - r * d), s);
    }
}

// ---- workspace ----------------------------------------------------------------------------------------------------
inline size_t pad256(size_t v) { return (v + 255) / 256 * 256; }

struct Plan {
    int planes, pack_w;
    int32_t ld, parts, width, pieces, dx_splits, dw_splits;
    int64_t Tpad;
    bool dx_slots, dw_slots;
    size_t o_live, o_scales, o_max, o_rows, o_x, o_w, o_idx, o_p, o_flags, o_teacher, o_part, o_dz, o_col, o_dx, o_dw, total;
};

// Tile counts follow from the sizes alone; how many tokens are kept is known on the device only.
Plan make_plan(int64_t T, int32_t d, int32_t V, int dtype, int32_t K, bool backward, bool dx_bf16)
{
    Plan p = {};
    p.planes = dtype == TBN_F32 ? 2 : 1;
    p.ld = (d + 7) / 8 * 8;
    p.pack_w = dtype == TBN_F32 || d % 8 != 0;
    p.Tpad = round_up64(T, kTile);
    const int64_t Vpad = round_up64(V, kTile);
    p.parts = (int32_t)(Vpad / kStatCols);
    size_t o = 0;
    auto take = [&o](size_t bytes) { const size_t at = o; o += pad256(bytes); return at; };
    p.o_live = take(4);
    p.o_scales = take(sizeof(Scales));
    p.o_max = take(12);
    p.o_rows = take((size_t)p.Tpad * sizeof(RowInfo));
    p.o_x = take((size_t)p.planes * p.Tpad * p.ld * 2);
    p.o_w = take(p.pack_w ? (size_t)p.planes * V * p.ld * 2 : 0);
    p.o_idx = take((size_t)T * K * 4);
    p.o_p = take((size_t)T * K * 4);
    p.o_flags = take(K > 0 ? (size_t)T : 0);
    p.o_teacher = take(K > 0 ? (size_t)T * 8 : 0);
    if (!backward) {
        p.o_part = take((size_t)3 * p.parts * p.Tpad * 4);
    } else {
        int64_t width = (int64_t)(kPieceBytes / ((size_t)2 * p.planes * p.Tpad)) / kTile * kTile;
        if (width < 1024) width = 1024;
        if (width > Vpad) width = Vpad;
        p.pieces = (int32_t)((Vpad + width - 1) / width);
        p.width = (int32_t)round_up64((Vpad + p.pieces - 1) / p.pieces, kTile);
        p.pieces = (int32_t)((Vpad + p.width - 1) / p.width);
        // a contraction is split when its few tiles would outlast the rest of the launch: no item longer than half of
        // an SM pair's even share of the work, or 8 steps
        const int64_t nt = (d + kTile - 1) / kTile, mt = p.Tpad / kTile, vt = p.width / kTile;
        const int64_t kx = p.width / 64, kw = (T + 63) / 64;
        const int64_t work = mt * nt * kx + vt * nt * kw;
        int64_t most = work / (2 * 74);
        if (most < 8) most = 8;
        auto splits = [most](int64_t k) { const int64_t s = (k + most - 1) / most; return (int32_t)(s < 1 ? 1 : s > kMaxSplits ? kMaxSplits : s); };
        p.dx_splits = splits(kx);
        p.dw_splits = splits(kw);
        p.dx_slots = p.dx_splits > 1 || (p.pieces > 1 && dx_bf16);
        p.dw_slots = p.dw_splits > 1;
        p.o_dz = take((size_t)p.planes * p.Tpad * p.width * 2);
        p.o_col = take((size_t)(p.Tpad / 32) * p.width * 4);
        p.o_dx = take(p.dx_slots ? (size_t)p.dx_splits * p.Tpad * d * 4 : 0);
        p.o_dw = take(p.dw_slots ? (size_t)p.dw_splits * p.width * d * 4 : 0);
    }
    p.total = o;
    return p;
}

unsigned blocks_for(int64_t items, int64_t per_block, int64_t most)
{
    int64_t b = (items + per_block - 1) / per_block;
    return (unsigned)(b < 1 ? 1 : b > most ? most : b);
}

// Labels, operands and per-row values: everything before the first contraction.
int prepare(const HeadCall &c, const Plan &p, char *ws, bool backward, LogitsArgs *out, cudaStream_t s)
{
    int32_t *n_live = reinterpret_cast<int32_t *>(ws + p.o_live);
    Scales *scales = reinterpret_cast<Scales *>(ws + p.o_scales);
    unsigned int *max_bits = reinterpret_cast<unsigned int *>(ws + p.o_max);
    RowInfo *rows = reinterpret_cast<RowInfo *>(ws + p.o_rows);
    const bool f32 = c.dtype == TBN_F32;
    Labels labels = {c.targets, c.ignore_index, c.V, nullptr};

    if (c.K > 0) {
        int32_t Kp = 32;
        while (Kp < c.K) Kp <<= 1;
        const size_t smem = (size_t)kTeacherWarps * Kp * 12;
        const dim3 grid((unsigned)((c.T + kTeacherWarps - 1) / kTeacherWarps));
        int32_t *idx = reinterpret_cast<int32_t *>(ws + p.o_idx);
        float *prob = reinterpret_cast<float *>(ws + p.o_p);
        uint8_t *flags = reinterpret_cast<uint8_t *>(ws + p.o_flags);
        float2 *stats = reinterpret_cast<float2 *>(ws + p.o_teacher);
        const cudaError_t e = c.top_dtype == TBN_F32
            ? launch_pdl(teacher_kernel<float>, grid, dim3(32 * kTeacherWarps), smem, s, c.top_index, static_cast<const float *>(c.top_logit),
                         c.T, c.K, Kp, c.V, 1.0f / c.tau, idx, prob, flags, stats)
            : launch_pdl(teacher_kernel<__nv_bfloat16>, grid, dim3(32 * kTeacherWarps), smem, s, c.top_index,
                         static_cast<const __nv_bfloat16 *>(c.top_logit), c.T, c.K, Kp, c.V, 1.0f / c.tau, idx, prob, flags, stats);
        if (e != cudaSuccess) return TBN_ERR_CUDA;
        labels.flags = flags;
        labels.target = nullptr;
        out->list_idx = idx;
        out->list_p = prob;
        out->K = c.K;
    }
    if (f32) {
        if (cudaMemsetAsync(max_bits, 0, 12, s) != cudaSuccess) return TBN_ERR_CUDA;
        const int64_t count = (int64_t)c.V * c.d;
        abs_max_kernel<<<blocks_for(count > c.T * c.d ? count : c.T * c.d, 4096, 1184), 256, 0, s>>>(
            static_cast<const float *>(c.x), labels, c.T, c.d, static_cast<const float *>(c.w), count, backward ? c.dloss : nullptr, c.tau, max_bits);
        if (cudaGetLastError() != cudaSuccess) return TBN_ERR_CUDA;
    }
    if (p.pack_w) {
        const unsigned grid = blocks_for((int64_t)c.V * (p.ld / 8), 256, 2368);
        uint16_t *wp = reinterpret_cast<uint16_t *>(ws + p.o_w);
        const cudaError_t e = f32
            ? launch_pdl(pack_weight_kernel<float>, dim3(grid), dim3(256), 0, s, static_cast<const float *>(c.w), (int64_t)c.V, c.d, p.ld, max_bits, wp)
            : launch_pdl(pack_weight_kernel<__nv_bfloat16>, dim3(grid), dim3(256), 0, s, static_cast<const __nv_bfloat16 *>(c.w), (int64_t)c.V, c.d,
                         p.ld, max_bits, wp);
        if (e != cudaSuccess) return TBN_ERR_CUDA;
    }
    PackArgs a = {};
    a.labels = labels; a.T = c.T; a.Tpad = p.Tpad; a.d = c.d; a.ld = p.ld;
    a.per_block = (c.T + 591) / 592 < 8 ? 8 : (c.T + 591) / 592;
    const unsigned blocks = (unsigned)((c.T + a.per_block - 1) / a.per_block);      // the last block has rows of its own
    a.max_bits = max_bits; a.xc = reinterpret_cast<uint16_t *>(ws + p.o_x); a.rows = rows; a.n_live = n_live; a.scales = scales; a.tau = c.tau;
    if (backward) {
        a.lse = c.lse; a.dloss = c.dloss; a.dx = c.dx; a.dx_bytes = c.dx_dtype == TBN_F32 ? 4 : 2;
    } else {
        a.loss_out = c.loss_out; a.lse_out = c.lse_out;
    }
    const cudaError_t e = f32 ? launch_pdl(pack_rows_kernel<float>, dim3(blocks), dim3(256), 0, s, static_cast<const float *>(c.x), a)
                              : launch_pdl(pack_rows_kernel<__nv_bfloat16>, dim3(blocks), dim3(256), 0, s, static_cast<const __nv_bfloat16 *>(c.x), a);
    if (e != cudaSuccess) return TBN_ERR_CUDA;

    out->x = Operand{ws + p.o_x, p.Tpad, p.Tpad, p.ld, p.ld};
    out->w = Operand{p.pack_w ? static_cast<const void *>(ws + p.o_w) : c.w, c.V, c.V, p.ld, p.ld};
    out->planes = p.planes;
    out->n_live = n_live; out->rows = rows; out->scales = f32 ? scales : nullptr;
    out->bias = c.bias; out->scale2 = kLog2e / c.tau; out->T = c.T; out->Tpad = p.Tpad; out->V = c.V;
    out->status = c.status;
    return TBN_OK;
}

}  // namespace

size_t workspace_bytes(int64_t T, int32_t d, int32_t V, int dtype, int32_t K, bool backward)
{
    return make_plan(T, d, V, dtype, K, backward, true).total;
}

int forward(const HeadCall &c, void *workspace, cudaStream_t s)
{
    const Plan p = make_plan(c.T, c.d, c.V, c.dtype, c.K, false, true);
    char *ws = static_cast<char *>(workspace);
    LogitsArgs a = {};
    int rc = prepare(c, p, ws, false, &a, s);
    if (rc != TBN_OK) return rc;
    a.v0 = 0; a.width = c.V;
    a.part_max = reinterpret_cast<float *>(ws + p.o_part);
    a.part_sum = a.part_max + (size_t)p.parts * p.Tpad;
    a.part_dot = a.part_sum + (size_t)p.parts * p.Tpad;
    rc = launch_head_stats(a, s);
    if (rc != TBN_OK) return rc;
    const float2 *teacher = c.K > 0 ? reinterpret_cast<const float2 *>(ws + p.o_teacher) : nullptr;
    // enough blocks for the GPU: one row per block when there are few tokens
    const int rb = c.T >= 4096 ? 32 : c.T >= 256 ? 8 : 1;
    const dim3 grid((unsigned)((c.T + rb - 1) / rb));
    auto kern = rb == 32 ? combine_kernel<32> : rb == 8 ? combine_kernel<8> : combine_kernel<1>;
    return launch_pdl(kern, grid, dim3(256), 0, s, a.part_max, a.part_sum, a.part_dot, p.parts, p.Tpad, a.n_live, a.rows, teacher, c.tau,
                      c.loss_out, c.lse_out) == cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
}

int backward(const HeadCall &c, void *workspace, cudaStream_t s)
{
    const bool dx_bf16 = c.dx_dtype == TBN_BF16;
    const Plan p = make_plan(c.T, c.d, c.V, c.dtype, c.K, true, dx_bf16);
    char *ws = static_cast<char *>(workspace);
    LogitsArgs a = {};
    int rc = prepare(c, p, ws, true, &a, s);
    if (rc != TBN_OK) return rc;
    a.dz = ws + p.o_dz;
    a.ldz = p.width;
    a.col_part = c.db ? reinterpret_cast<float *>(ws + p.o_col) : nullptr;

    GradArgs g = {};
    g.x = a.x; g.w = a.w; g.planes = a.planes; g.n_live = a.n_live; g.rows = a.rows; g.scales = a.scales; g.dz = a.dz;
    g.T = c.T; g.Tpad = p.Tpad; g.d = c.d; g.V = c.V; g.ldz = p.width;
    g.want_dx = c.dx != nullptr; g.want_dw = c.dw != nullptr;
    g.dx = c.dx; g.dx_bf16 = dx_bf16; g.dx_slots = p.dx_slots ? reinterpret_cast<float *>(ws + p.o_dx) : nullptr; g.dx_splits = p.dx_splits;
    g.dw = c.dw; g.dw_bf16 = c.dw_dtype == TBN_BF16; g.dw_slots = p.dw_slots ? reinterpret_cast<float *>(ws + p.o_dw) : nullptr;
    g.dw_splits = p.dw_splits;
    g.status = c.status;
    for (int32_t piece = 0; piece < p.pieces; ++piece) {
        a.v0 = piece * p.width;
        a.width = c.V - a.v0 < p.width ? c.V - a.v0 : p.width;
        rc = launch_head_dz(a, s);
        if (rc != TBN_OK) return rc;
        if (c.db && launch_pdl(bias_grad_kernel, dim3((unsigned)((a.width + 31) / 32)), dim3(256), 0, s, static_cast<const float *>(a.col_part), a.ldz,
                               a.n_live, a.scales, a.width, c.db + a.v0) != cudaSuccess)
            return TBN_ERR_CUDA;
        if (!g.want_dx && !g.want_dw) continue;
        g.v0 = a.v0; g.width = a.width;
        g.dx_add = piece > 0;
        g.dx_last = piece == p.pieces - 1;
        rc = launch_head_grads(g, s);
        if (rc != TBN_OK) return rc;
        if (g.want_dw && p.dw_splits > 1) {
            const int64_t rows = a.width;
            const unsigned grid = blocks_for(rows * c.d, 1024, 1184);
            const int64_t slot_rows = round_up64(a.width, kTile);
            const RowInfo *none = nullptr;
            const cudaError_t e = g.dw_bf16
                ? launch_pdl(join_splits_kernel<__nv_bfloat16>, dim3(grid), dim3(256), 0, s, static_cast<const float *>(g.dw_slots), p.dw_splits, slot_rows,
                             c.d, a.n_live, none, rows, static_cast<__nv_bfloat16 *>(c.dw) + (int64_t)a.v0 * c.d)
                : launch_pdl(join_splits_kernel<float>, dim3(grid), dim3(256), 0, s, static_cast<const float *>(g.dw_slots), p.dw_splits, slot_rows, c.d,
                             a.n_live, none, rows, static_cast<float *>(c.dw) + (int64_t)a.v0 * c.d);
            if (e != cudaSuccess) return TBN_ERR_CUDA;
        }
    }
    if (g.want_dx && p.dx_splits > 1) {
        const unsigned grid = blocks_for(c.T * c.d, 1024, 1184);
        const cudaError_t e = dx_bf16
            ? launch_pdl(join_splits_kernel<__nv_bfloat16>, dim3(grid), dim3(256), 0, s, static_cast<const float *>(g.dx_slots), p.dx_splits, p.Tpad, c.d,
                         a.n_live, a.rows, (int64_t)0, static_cast<__nv_bfloat16 *>(c.dx))
            : launch_pdl(join_splits_kernel<float>, dim3(grid), dim3(256), 0, s, static_cast<const float *>(g.dx_slots), p.dx_splits, p.Tpad, c.d, a.n_live,
                         a.rows, (int64_t)0, static_cast<float *>(c.dx));
        if (e != cudaSuccess) return TBN_ERR_CUDA;
    }
    return TBN_OK;
}

}  // namespace head
}  // namespace tbn
