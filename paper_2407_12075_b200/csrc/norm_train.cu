// LayerNorm for training: the forward with an optional residual input that keeps a row's mean and 1 / standard deviation, and the
// backward with the sums over rows that the gains and offsets need.
//
//   s = x + residual,  h = (s - mean) rstd,  y = h gamma + beta
//   a = dy gamma,  ds = rstd (a - mean(a) - h mean(a h)) (+ dsum),  dgamma = sum_t dy h,  dbeta = sum_t dy
//
// Both are bound by HBM: each row is read once and held in registers, and the columns' sums stay in registers over all rows of
// a thread block.
#include <atomic>

#include "norm_train.cuh"
#include "vec8.cuh"

namespace tbn {
namespace norm {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxWarps = 8;                // warps that share a row at most

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}
// Threads of one row group meet; a group of one warp needs no barrier of its own.
__device__ __forceinline__ void group_sync(int group, int threads)
{
    if (threads == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" :: "r"(group + 1), "r"(threads) : "memory");
}

// Columns of a thread in a row group of `threads`: pieces of eight in a row (VEC) or single columns, NP * 8 in all.
template <bool VEC> __device__ __forceinline__ int32_t column(int i, int e, int tid, int threads)
{
    return VEC ? (i * threads + tid) * 8 + e : (i * 8 + e) * threads + tid;
}
template <bool VEC, typename T> __device__ __forceinline__ void load_piece(const T *row, int i, int tid, int threads, int32_t d, float (&v)[8])
{
    if (VEC) {
        const int32_t c = column<true>(i, 0, tid, threads);
        if (c < d) unpack8(load8(row + c), v);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.0f;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int32_t c = column<false>(i, e, tid, threads);
            v[e] = c < d ? value_of(row[c]) : 0.0f;
        }
    }
}
template <bool VEC, typename T> __device__ __forceinline__ void store_piece(T *row, int i, int tid, int threads, int32_t d, const float (&v)[8])
{
    if (VEC) {
        const int32_t c = column<true>(i, 0, tid, threads);
        if (c < d) store8(row + c, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int32_t c = column<false>(i, e, tid, threads);
            if (c < d) store_from_float(row, c, v[e]);
        }
    }
}

template <typename XT> __device__ __forceinline__ float rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ float rounded<__nv_bfloat16>(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

// One row to a group of `warps` warps.  The mean and the centred second moment are taken per warp and joined over the warps
// (two sets of n1 and n2 values: M2 = M2a + M2b + (mean_b - mean_a)^2 n1 n2 / (n1 + n2)), so that a group meets once a row.
template <typename XT, typename YT, int NP, bool VEC>
__global__ void __launch_bounds__(kThreads)
forward_kernel(const XT *__restrict__ x, const XT *__restrict__ residual, int64_t T, int32_t d, int warps, const float *__restrict__ gamma,
               const float *__restrict__ beta, float eps, XT *__restrict__ sum, YT *__restrict__ y, float *__restrict__ mean_out,
               float *__restrict__ rstd_out)
{
    __shared__ float3 part[kMaxWarps];
    pdl_launch_dependents();
    pdl_wait();
    const int threads = warps * 32, group = threadIdx.x / threads, tid = threadIdx.x - group * threads;
    const int64_t t = (int64_t)blockIdx.x * (blockDim.x / threads) + group;
    if (t >= T) return;                                               // a whole group
    float v[NP][8];
#pragma unroll
    for (int i = 0; i < NP; ++i) load_piece<VEC>(x + t * d, i, tid, threads, d, v[i]);
    if (residual) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            float r[8];
            load_piece<VEC>(residual + t * d, i, tid, threads, d, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = rounded<XT>(v[i][e] + r[e]);
            if (sum) store_piece<VEC>(sum + t * d, i, tid, threads, d, v[i]);
        }
    }
    float s = 0.0f;
    int32_t mine = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) { s += v[i][e]; mine += column<VEC>(i, e, tid, threads) < d; }
    float n = warps == 1 ? (float)d : (float)__reduce_add_sync(0xffffffffu, mine);
    float mean = n > 0.0f ? warp_sum(s) / n : 0.0f;
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (column<VEC>(i, e, tid, threads) < d) { const float c = v[i][e] - mean; q = fmaf(c, c, q); }
    q = warp_sum(q);
    if (warps > 1) {
        const int first = group * warps;
        if ((tid & 31) == 0) part[first + (tid >> 5)] = make_float3(n, mean, q);
        group_sync(group, threads);
        n = part[first].x; mean = part[first].y; q = part[first].z;
        for (int w = 1; w < warps; ++w) {
            const float3 b = part[first + w];
            if (b.x > 0.0f) {
                const float both = n + b.x, delta = b.y - mean, share = b.x / both;
                mean = fmaf(delta, share, mean);
                q += fmaf(delta * delta, n * share, b.z);
                n = both;
            }
        }
    }
    const float rstd = rsqrtf(q / (float)d + eps);
    if (tid == 0) {
        if (mean_out) mean_out[t] = mean;
        if (rstd_out) rstd_out[t] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        float o[8], w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (v[i][e] - mean) * rstd;
        if (gamma) {
            load_piece<VEC>(gamma, i, tid, threads, d, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] *= w[e];
        }
        if (beta) {
            load_piece<VEC>(beta, i, tid, threads, d, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += w[e];
        }
        store_piece<VEC>(y + t * d, i, tid, threads, d, o);
    }
}

// Rows longer than a group's registers hold: three passes over a row, the second and third from the cache.
template <typename XT, typename YT>
__global__ void __launch_bounds__(kThreads)
forward_long_kernel(const XT *__restrict__ x, const XT *__restrict__ residual, int64_t T, int32_t d, const float *__restrict__ gamma,
                    const float *__restrict__ beta, float eps, XT *__restrict__ sum, YT *__restrict__ y, float *__restrict__ mean_out,
                    float *__restrict__ rstd_out)
{
    __shared__ float part[2][kThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    auto all = [&](float v, int which) {
        v = warp_sum(v);
        if ((threadIdx.x & 31) == 0) part[which][threadIdx.x >> 5] = v;
        __syncthreads();
        float t = 0.0f;
        for (int w = 0; w < kThreads / 32; ++w) t += part[which][w];
        return t;
    };
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
        auto at = [&](int32_t c) { return residual ? rounded<XT>(value_of(x[t * d + c]) + value_of(residual[t * d + c])) : value_of(x[t * d + c]); };
        float s = 0.0f;
        for (int32_t c = threadIdx.x; c < d; c += kThreads) s += at(c);
        const float mean = all(s, 0) / (float)d;
        float q = 0.0f;
        for (int32_t c = threadIdx.x; c < d; c += kThreads) { const float e = at(c) - mean; q = fmaf(e, e, q); }
        const float rstd = rsqrtf(all(q, 1) / (float)d + eps);
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[t] = mean;
            if (rstd_out) rstd_out[t] = rstd;
        }
        for (int32_t c = threadIdx.x; c < d; c += kThreads) {
            const float v = at(c);
            float o = (v - mean) * rstd;
            if (gamma) o *= gamma[c];
            if (beta) o += beta[c];
            if (residual && sum) store_from_float(sum + t * d, c, v);
            store_from_float(y + t * d, c, o);
        }
    }
}

// A thread block walks over rows with a stride; a thread keeps its columns' share of dgamma and dbeta in registers to the end.
template <typename XT, typename YT, int NP, bool VEC>
__global__ void __launch_bounds__(kThreads)
backward_kernel(const YT *__restrict__ dy, const XT *__restrict__ x, int64_t T, int32_t d, int warps, const float *__restrict__ gamma,
                const float *__restrict__ mean, const float *__restrict__ rstd, const XT *__restrict__ dsum, XT *__restrict__ dx,
                float *__restrict__ partial)
{
    __shared__ float2 part[2][kMaxWarps];
    extern __shared__ float columns[];                                // with several groups: [groups][2][d]
    pdl_launch_dependents();
    pdl_wait();
    const int threads = warps * 32, group = threadIdx.x / threads, tid = threadIdx.x - group * threads;
    const int groups = blockDim.x / threads;
    float dg[NP][8], db[NP][8], w[NP][8];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { dg[i][e] = db[i][e] = 0.0f; w[i][e] = 1.0f; }
        if (gamma) load_piece<VEC>(gamma, i, tid, threads, d, w[i]);
    }
    const float inv_d = 1.0f / (float)d;
    int turn = 0;
    for (int64_t t = (int64_t)blockIdx.x * groups + group; t < T; t += (int64_t)gridDim.x * groups, turn ^= 1) {
        float g[NP][8], h[NP][8];
        const float mu = mean[t], rs = rstd[t];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            load_piece<VEC>(dy + t * d, i, tid, threads, d, g[i]);
            load_piece<VEC>(x + t * d, i, tid, threads, d, h[i]);
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                h[i][e] = (h[i][e] - mu) * rs;                        // beyond the row: times a g of zero
                db[i][e] += g[i][e];
                dg[i][e] = fmaf(g[i][e], h[i][e], dg[i][e]);
                g[i][e] *= w[i][e];
                s1 += g[i][e];
                s2 = fmaf(g[i][e], h[i][e], s2);
            }
        s1 = warp_sum(s1); s2 = warp_sum(s2);
        if (warps > 1) {
            const int first = group * warps;
            if ((tid & 31) == 0) part[turn][first + (tid >> 5)] = make_float2(s1, s2);
            group_sync(group, threads);
            s1 = s2 = 0.0f;
            for (int k = 0; k < warps; ++k) { s1 += part[turn][first + k].x; s2 += part[turn][first + k].y; }
        }
        s1 *= inv_d; s2 *= inv_d;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            float r[8];
            if (dsum) load_piece<VEC>(dsum + t * d, i, tid, threads, d, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float o = (g[i][e] - s1 - h[i][e] * s2) * rs;
                g[i][e] = dsum ? o + r[e] : o;
            }
            store_piece<VEC>(dx + t * d, i, tid, threads, d, g[i]);
        }
    }
    if (!partial) return;
    float *out = partial + (int64_t)blockIdx.x * 2 * d;
    if (groups == 1) {
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int32_t c = column<VEC>(i, e, tid, threads);
                if (c < d) { out[c] = dg[i][e]; out[d + c] = db[i][e]; }
            }
        return;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int32_t c = column<VEC>(i, e, tid, threads);
            if (c < d) { columns[group * 2 * d + c] = dg[i][e]; columns[group * 2 * d + d + c] = db[i][e]; }
        }
    __syncthreads();
    for (int32_t c = threadIdx.x; c < 2 * d; c += blockDim.x) {
        float t = columns[c];
        for (int k = 1; k < groups; ++k) t += columns[k * 2 * d + c];
        out[c] = t;
    }
}

// Rows longer than a group's registers hold: two passes over a row, and the columns' sums by thread blocks of their own.
template <typename XT, typename YT>
__global__ void __launch_bounds__(kThreads)
backward_long_kernel(const YT *__restrict__ dy, const XT *__restrict__ x, int64_t T, int32_t d, const float *__restrict__ gamma,
                     const float *__restrict__ mean, const float *__restrict__ rstd, const XT *__restrict__ dsum, XT *__restrict__ dx)
{
    __shared__ float2 part[2][kThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    int turn = 0;
    for (int64_t t = blockIdx.x; t < T; t += gridDim.x, turn ^= 1) {
        const float mu = mean[t], rs = rstd[t];
        float s1 = 0.0f, s2 = 0.0f;
        for (int32_t c = threadIdx.x; c < d; c += kThreads) {
            const float a = value_of(dy[t * d + c]) * (gamma ? gamma[c] : 1.0f);
            s1 += a;
            s2 = fmaf(a, (value_of(x[t * d + c]) - mu) * rs, s2);
        }
        s1 = warp_sum(s1); s2 = warp_sum(s2);
        if ((threadIdx.x & 31) == 0) part[turn][threadIdx.x >> 5] = make_float2(s1, s2);
        __syncthreads();
        s1 = s2 = 0.0f;
        for (int k = 0; k < kThreads / 32; ++k) { s1 += part[turn][k].x; s2 += part[turn][k].y; }
        s1 /= (float)d; s2 /= (float)d;
        for (int32_t c = threadIdx.x; c < d; c += kThreads) {
            const float a = value_of(dy[t * d + c]) * (gamma ? gamma[c] : 1.0f);
            float o = (a - s1 - (value_of(x[t * d + c]) - mu) * rs * s2) * rs;
            if (dsum) o += value_of(dsum[t * d + c]);
            store_from_float(dx + t * d, c, o);
        }
    }
}
template <typename XT, typename YT>
__global__ void __launch_bounds__(kThreads)
column_sums_kernel(const YT *__restrict__ dy, const XT *__restrict__ x, int64_t T, int32_t d, const float *__restrict__ mean,
                   const float *__restrict__ rstd, float *__restrict__ partial)
{
    pdl_launch_dependents();
    pdl_wait();
    float *out = partial + (int64_t)blockIdx.y * 2 * d;
    for (int32_t c = blockIdx.x * kThreads + threadIdx.x; c < d; c += gridDim.x * kThreads) {
        float dg = 0.0f, db = 0.0f;
        for (int64_t t = blockIdx.y; t < T; t += gridDim.y) {
            const float g = value_of(dy[t * d + c]);
            db += g;
            dg = fmaf(g, (value_of(x[t * d + c]) - mean[t]) * rstd[t], dg);
        }
        out[c] = dg;
        out[d + c] = db;
    }
}

// Adds the thread blocks' sums in a fixed order: 32 columns to a block, 8 rows of them at a time.
__global__ void __launch_bounds__(kThreads)
finish_kernel(const float *__restrict__ partial, int32_t parts, int32_t d, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    __shared__ float red[kThreads / 32][32];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;                // of dgamma's d and dbeta's d
    float t = 0.0f;
    if (c < 2 * (int64_t)d)
        for (int32_t k = row; k < parts; k += kThreads / 32) t += partial[(int64_t)k * 2 * d + c];
    red[row][lane] = t;
    __syncthreads();
    if (row == 0 && c < 2 * (int64_t)d) {
#pragma unroll
        for (int k = 1; k < kThreads / 32; ++k) t += red[k][lane];
        if (c < d) { if (dgamma) dgamma[c] = t; }
        else if (dbeta) dbeta[c - d] = t;
    }
}

int sm_count()
{
    static std::atomic<int> cache[64];
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
    n = cache[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 148;
        cache[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

struct Shape {
    int np, warps, groups;                  // pieces of eight columns to a thread, warps to a row, rows to a thread block
    bool vec, lng;
};
Shape shape_of(int32_t d, bool vec)
{
    Shape s;
    s.vec = vec;
    s.lng = d > kThreads * 8 * 4;
    s.np = d <= kThreads * 8 ? 1 : d <= kThreads * 16 ? 2 : 4;
    s.warps = (d + 256 * s.np - 1) / (256 * s.np);
    s.groups = kMaxWarps / s.warps;
    return s;
}
// Thread blocks of the backward pass: what fits on the GPU at a time, and no more than there are rows.
int64_t backward_blocks(int64_t T, const Shape &s)
{
    const int64_t most = (int64_t)sm_count() * 2, need = (T + s.groups - 1) / s.groups;
    return need < most ? need : most;
}
constexpr int kLongParts = 64;

template <typename F> cudaError_t with_shape(const Shape &s, F f)
{
    if (s.vec) return s.np == 1 ? f(std::integral_constant<int, 1>{}, std::true_type{}) : s.np == 2 ? f(std::integral_constant<int, 2>{}, std::true_type{})
                                                                                       : f(std::integral_constant<int, 4>{}, std::true_type{});
    return s.np == 1 ? f(std::integral_constant<int, 1>{}, std::false_type{}) : s.np == 2 ? f(std::integral_constant<int, 2>{}, std::false_type{})
                                                                                  : f(std::integral_constant<int, 4>{}, std::false_type{});
}

template <typename XT, typename YT> cudaError_t forward_typed(const ForwardArgs &a, cudaStream_t s)
{
    const bool vec = aligned8<XT>(a.x, a.d) && aligned8<XT>(a.residual) && aligned8<XT>(a.sum) && aligned8<YT>(a.y) && aligned8<float>(a.gamma) &&
                     aligned8<float>(a.beta);
    const Shape sh = shape_of(a.d, vec);
    const XT *x = static_cast<const XT *>(a.x), *r = static_cast<const XT *>(a.residual);
    XT *sum = static_cast<XT *>(a.sum);
    YT *y = static_cast<YT *>(a.y);
    if (sh.lng) {
        const int64_t most = (int64_t)sm_count() * 8;
        return launch_pdl(forward_long_kernel<XT, YT>, dim3((unsigned)(a.T < most ? a.T : most)), dim3(kThreads), 0, s, x, r, a.T, a.d, a.gamma,
                          a.beta, a.eps, sum, y, a.mean, a.rstd);
    }
    return with_shape(sh, [&](auto np, auto v) {
        return launch_pdl(forward_kernel<XT, YT, decltype(np)::value, decltype(v)::value>, dim3((unsigned)((a.T + sh.groups - 1) / sh.groups)),
                          dim3(sh.groups * sh.warps * 32), 0, s, x, r, a.T, a.d, sh.warps, a.gamma, a.beta, a.eps, sum, y, a.mean, a.rstd);
    });
}

template <typename XT, typename YT> cudaError_t backward_typed(const BackwardArgs &a, float *partial, cudaStream_t s)
{
    const bool vec = aligned8<XT>(a.x, a.d) && aligned8<YT>(a.dy) && aligned8<XT>(a.dsum) && aligned8<XT>(a.dx) && aligned8<float>(a.gamma);
    const Shape sh = shape_of(a.d, vec);
    const YT *dy = static_cast<const YT *>(a.dy);
    const XT *x = static_cast<const XT *>(a.x), *dsum = static_cast<const XT *>(a.dsum);
    XT *dx = static_cast<XT *>(a.dx);
    const bool sums = a.dgamma || a.dbeta;
    int32_t parts;
    cudaError_t e;
    if (sh.lng) {
        const int64_t most = (int64_t)sm_count() * 8;
        e = launch_pdl(backward_long_kernel<XT, YT>, dim3((unsigned)(a.T < most ? a.T : most)), dim3(kThreads), 0, s, dy, x, a.T, a.d, a.gamma,
                       a.mean, a.rstd, dsum, dx);
        parts = (int32_t)(a.T < kLongParts ? a.T : kLongParts);
        const int32_t slabs = (a.d + kThreads - 1) / kThreads;
        if (e == cudaSuccess && sums)
            e = launch_pdl(column_sums_kernel<XT, YT>, dim3(slabs < 4096 ? slabs : 4096, parts), dim3(kThreads), 0, s, dy, x, a.T, a.d, a.mean,
                           a.rstd, partial);
    } else {
        parts = (int32_t)backward_blocks(a.T, sh);
        const size_t smem = sh.groups > 1 ? (size_t)sh.groups * 2 * a.d * 4 : 0;       // at most 8 x 2 x 256 floats' worth
        e = with_shape(sh, [&](auto np, auto v) {
            return launch_pdl(backward_kernel<XT, YT, decltype(np)::value, decltype(v)::value>, dim3((unsigned)parts),
                              dim3(sh.groups * sh.warps * 32), smem, s, dy, x, a.T, a.d, sh.warps, a.gamma, a.mean, a.rstd, dsum, dx,
                              sums ? partial : nullptr);
        });
    }
    if (e != cudaSuccess || !sums) return e;
    return launch_pdl(finish_kernel, dim3((unsigned)((2 * (int64_t)a.d + 31) / 32)), dim3(kThreads), 0, s, static_cast<const float *>(partial), parts,
                      a.d, a.dgamma, a.dbeta);
}

}  // namespace

size_t backward_workspace_bytes(int64_t T, int32_t d)
{
    const Shape sh = shape_of(d, true);
    const int64_t parts = sh.lng ? (T < kLongParts ? T : kLongParts) : backward_blocks(T, sh);
    return (size_t)parts * 2 * (size_t)d * 4;
}

int forward(const ForwardArgs &a, cudaStream_t s)
{
    cudaError_t e;
    if (a.x_dtype == TBN_F32) e = a.y_dtype == TBN_F32 ? forward_typed<float, float>(a, s) : forward_typed<float, __nv_bfloat16>(a, s);
    else e = a.y_dtype == TBN_F32 ? forward_typed<__nv_bfloat16, float>(a, s) : forward_typed<__nv_bfloat16, __nv_bfloat16>(a, s);
    return e == cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
}

int backward(const BackwardArgs &a, void *workspace, cudaStream_t s)
{
    float *partial = static_cast<float *>(workspace);
    cudaError_t e;
    if (a.x_dtype == TBN_F32) e = a.dy_dtype == TBN_F32 ? backward_typed<float, float>(a, partial, s) : backward_typed<float, __nv_bfloat16>(a, partial, s);
    else e = a.dy_dtype == TBN_F32 ? backward_typed<__nv_bfloat16, float>(a, partial, s) : backward_typed<__nv_bfloat16, __nv_bfloat16>(a, partial, s);
    return e == cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
}

}  // namespace norm
}  // namespace tbn
