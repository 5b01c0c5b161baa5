// LayerNorm for training: the forward with an optional residual input that keeps a row's mean and 1 / standard deviation, and the
// backward with the sums over rows that the gains and offsets need.
//
//   s = x + residual,  h = (s - mean) rstd,  y = h gamma + beta
//   a = dy gamma,  ds = rstd (a - mean(a) - h mean(a h)) (+ dsum),  dgamma = sum_t dy h,  dbeta = sum_t dy
//
// Both are bound by HBM: each row is read once, through a ring in shared memory that asynchronous copies fill (so that the next
// rows are on their way while one is worked on), and held in registers; the columns' sums stay in registers over all rows of a thread
// block.  A row is shared by 1 to 8 warps, a lane has 1 to 4 pieces of eight columns; rows of up to 128 columns have 4, 8 or 16 lanes each
// of a warp that works on several.
//
// Rows that do not begin on 16 bytes are read and written as the aligned pieces that cover them, what is not the row's being masked.
// Where a piece begins in a row then depends on the row, (t d) mod 8, so a thread block keeps to rows of one remainder, and a lane
// to its columns.
#include <atomic>
#include <type_traits>

#include "norm_train.cuh"
#include "vec8.cuh"

namespace tbn {
namespace norm {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxWarps = 8;                // warps that share a row at most

// Sum over groups of SUB lanes.
template <int SUB = 32> __device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int off = SUB / 2; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}
// Threads of one row group meet; a group of one warp needs no barrier of its own.
__device__ __forceinline__ void group_sync(int group, int threads)
{
    if (threads == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" :: "r"(group + 1), "r"(threads) : "memory");
}

template <typename XT> __device__ __forceinline__ float rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ float rounded<__nv_bfloat16>(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

// How a call's rows and columns are spread over thread blocks, warps and lanes.
struct Shape {
    int np, warps, groups;                  // pieces of eight columns to a lane, warps to a row, rows to a thread block
    int sub;                                // lanes to a row: 32, or 4, 8 or 16 of narrow rows, several of which a warp works on
    int classes;                            // remainders (t d) mod unit that occur: thread block b takes rows t = b mod classes
    bool lng;
};

// What a lane has to do with the rows of its group.  EVEN: d is a multiple of eight, so that rows begin and end with whole pieces.
template <int NP, bool EVEN, int SUB> struct Lane {
    int32_t shift;                          // columns between the aligned piece that a row begins in and the row
    int threads, group, lane;               // threads of a row's group; lane of the warp
    bool first;                             // of the group's lanes
    int32_t at;                             // the lane's first column from the aligned start on; its next pieces are 256 columns apart
    int64_t row, row_step, rows;            // first row, from one to the next, how many
    int64_t total;                          // elements of the whole tensor
    uint32_t mask[NP];                      // which of a piece's eight columns are the row's
    uint32_t edges;                         // pieces of which a lane of the warp has a part
    __device__ __forceinline__ Lane(int64_t T, int32_t d, int warps, int groups, int classes)
    {
        threads = SUB < 32 ? SUB : warps * 32;
        group = threadIdx.x / threads;
        lane = threadIdx.x & 31;
        const int in_group = threadIdx.x - group * threads;
        first = in_group == 0;
        at = SUB < 32 ? in_group * 8 : ((in_group >> 5) * NP * 32 + lane) * 8;
        const int cls = EVEN ? 0 : blockIdx.x % classes;
        const int64_t first = (int64_t)(EVEN ? blockIdx.x : blockIdx.x / classes) * groups + group, step = (int64_t)(gridDim.x / classes) * groups;
        const int64_t here = (T - cls + classes - 1) / classes;      // rows of the class
        rows = first < here ? (here - first - 1) / step + 1 : 0;
        row = cls + first * classes;
        row_step = step * classes;
        total = T * d;
        shift = EVEN ? 0 : (int32_t)(((int64_t)cls * d) & 7);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            mask[i] = 0;
            if (EVEN) mask[i] = at + i * 256 < d ? 0xffu : 0u;
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int32_t c = at + i * 256 + e - shift;
                    if (c >= 0 && c < d) mask[i] |= 1u << e;
                }
        }
        edges = 0;
        if (!EVEN) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
                if (__any_sync(0xffffffffu, mask[i] != 0 && mask[i] != 0xffu)) edges |= 1u << i;
        }
    }
};

// Ring of a warp in shared memory.  A lane copies and takes its own pieces, so that nothing but its own copies is waited for.
// start: of the row in x, plus the lane's first column.
template <typename T, int NP, bool EVEN, int SUB>
__device__ __forceinline__ void fetch(uint32_t to, const T *x, int64_t start, const Lane<NP, EVEN, SUB> &l)
{
    const T *from = x + start;
    constexpr int kPer = 16 / (int)sizeof(T);
    const bool whole = EVEN || start + (NP - 1) * 256 + 8 <= l.total;             // at the tensor's end a piece may be a part
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        if (l.mask[i] == 0) continue;
#pragma unroll
        for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
            const uint32_t slot = to + (i * ((int)sizeof(T) / 2) + h) * 512;
            const T *f = from + i * 256 + h * kPer;
            if (whole) {
                if (sizeof(T) == 2) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(slot), "l"(f) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" :: "r"(slot), "l"(f) : "memory");
            } else {                                                  // what is behind the end is not read
                const int64_t left = l.total - start - i * 256 - h * kPer;
                const int size = left >= kPer ? 16 : left > 0 ? (int)left * (int)sizeof(T) : 0;
                if (size == 0) f = x;
                if (sizeof(T) == 2) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(slot), "l"(f), "r"(size) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" :: "r"(slot), "l"(f), "r"(size) : "memory");
            }
        }
    }
}
// A piece's eight mask bits as the signs of eight bytes, which a byte permutation spreads over a value's bits.
struct Signs {
    uint32_t lo, hi;
    __device__ __forceinline__ explicit Signs(uint32_t mask)
        : lo((((mask & 15u) * 0x00204081u) & 0x01010101u) * 0x80u), hi((((mask >> 4) * 0x00204081u) & 0x01010101u) * 0x80u) {}
    template <uint32_t SELECT> static __device__ __forceinline__ uint32_t spread(uint32_t s)
    {
        uint32_t r;
        asm("prmt.b32 %0, %1, 0, %2;" : "=r"(r) : "r"(s), "n"(SELECT));
        return r;
    }
    __device__ __forceinline__ void keep(Raw8<__nv_bfloat16> &r) const
    {
        r.w[0] &= spread<0x9988>(lo); r.w[1] &= spread<0xbbaa>(lo);
        r.w[2] &= spread<0x9988>(hi); r.w[3] &= spread<0xbbaa>(hi);
    }
    __device__ __forceinline__ void keep(Raw8<float> &r) const
    {
        r.w[0] &= spread<0x8888>(lo); r.w[1] &= spread<0x9999>(lo); r.w[2] &= spread<0xaaaa>(lo); r.w[3] &= spread<0xbbbb>(lo);
        r.w[4] &= spread<0x8888>(hi); r.w[5] &= spread<0x9999>(hi); r.w[6] &= spread<0xaaaa>(hi); r.w[7] &= spread<0xbbbb>(hi);
    }
    __device__ __forceinline__ void keep(Pair (&v)[4]) const          // zero where there is no column
    {
        Raw8<float> r;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = split(v[e]);
            r.w[2 * e] = __float_as_uint(f.x); r.w[2 * e + 1] = __float_as_uint(f.y);
        }
        keep(r);
        unpack8(r, v);
    }
};
// Slots of pieces without columns hold zeros from the start on.
template <typename T, int NP, bool EVEN, int SUB> __device__ __forceinline__ void take(const char *from, int i, const Lane<NP, EVEN, SUB> &l, Pair (&v)[4])
{
    Raw8<T> r;
    const uint4 *q = reinterpret_cast<const uint4 *>(from + i * (int)sizeof(T) / 2 * 512);
#pragma unroll
    for (int h = 0; h < (int)sizeof(T) / 2; ++h) {
        const uint4 x = q[h * 32];
        r.w[4 * h] = x.x; r.w[4 * h + 1] = x.y; r.w[4 * h + 2] = x.z; r.w[4 * h + 3] = x.w;
    }
    if (!EVEN && (l.edges >> i & 1u)) Signs(l.mask[i]).keep(r);
    unpack8(r, v);
}
__device__ __forceinline__ void store16(float *p, const Pair (&v)[4])
{
    float f[8];
    spread8(v, f);
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store16(__nv_bfloat16 *p, const Pair (&v)[4])
{
    float f[8];
    spread8(v, f);
    store8(p, f);
}
template <typename T, int NP, bool EVEN, int SUB> __device__ __forceinline__ void put(T *x, int64_t start, int i, const Lane<NP, EVEN, SUB> &l, const Pair (&v)[4])
{
    T *p = x + start + i * 256;
    if (l.mask[i] == 0xffu) store16(p, v);
    else if (!EVEN && l.mask[i] != 0) {
        float f[8];
        spread8(v, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) if (l.mask[i] >> e & 1u) store_from_float(p, e, f[e]);
    }
}
// A vector of d floats (or ones) in shared memory, from the aligned start on, as the thread block's rows lie.
__device__ __forceinline__ void stage_vector(float *to, const float *from, float otherwise, int32_t d, int32_t shift, int32_t room)
{
    for (int32_t c = threadIdx.x; c < room; c += blockDim.x) to[c] = from && c >= shift && c - shift < d ? from[c - shift] : otherwise;
}
__device__ __forceinline__ void read8(const float *from, Pair (&v)[4])
{
    const float4 a = reinterpret_cast<const float4 *>(from)[0], b = reinterpret_cast<const float4 *>(from)[1];
    v[0] = pair(a.x, a.y); v[1] = pair(a.z, a.w); v[2] = pair(b.x, b.y); v[3] = pair(b.z, b.w);
}
template <typename XT> __device__ __forceinline__ void round8(Pair (&v)[4]);
template <> __device__ __forceinline__ void round8<float>(Pair (&)[4]) {}
template <> __device__ __forceinline__ void round8<__nv_bfloat16>(Pair (&v)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 f = split(v[e]);
        const uint32_t w = pack_bf16(f.x, f.y);
        v[e] = pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
}

// Rows in the ring: two thread blocks of eight warps to an SM, half its shared memory each, less what gains and offsets take there.
constexpr int stages_for(int row_bytes)     // of one warp
{
    const int s = 92 * 1024 / (kMaxWarps * row_bytes);
    return s < 2 ? 2 : s > 4 ? 4 : s;
}
template <typename XT, typename YT, int NP> struct ForwardRing {
    static constexpr int kX = NP * 256 * (int)sizeof(XT), kBytes = 2 * kX, kStages = stages_for(kBytes);
};
template <typename XT, typename YT, int NP> struct BackwardRing {
    static constexpr int kX = NP * 256 * (int)sizeof(XT), kY = NP * 256 * (int)sizeof(YT), kBytes = 2 * kX + kY, kStages = stages_for(kBytes);
};

// The mean and the centred second moment are taken per warp and joined over the warps of a row (of two sets of n1 and n2 values:
// M2 = M2a + M2b + (mean_b - mean_a)^2 n1 n2 / (n1 + n2)), so that a group meets once a row.  bf16 with a residual: 25216 x 768 in 27 us
// (5.7 TB/s), 8192 x 2048 in 25 us (5.4); a thread block for each few rows, gains and offsets read anew, took 62 and 52.
template <typename XT, typename YT, int NP, bool EVEN, int SUB>
__global__ void __launch_bounds__(kThreads, 2)
forward_kernel(const ForwardArgs a, const Shape sh)
{
    typedef ForwardRing<XT, YT, NP> R;
    __shared__ float3 part[2][kMaxWarps];
    extern __shared__ __align__(16) char smem[];
    pdl_launch_dependents();
    pdl_wait();
    const Lane<NP, EVEN, SUB> l(a.T, a.d, sh.warps, sh.groups, sh.classes);
    const int32_t room = SUB < 32 ? SUB * 8 : sh.warps * NP * 256;
    float *gamma = reinterpret_cast<float *>(smem) + l.at, *beta = gamma + room;
    char *ring = smem + 2 * room * 4 + (threadIdx.x >> 5) * (R::kStages * R::kBytes) + l.lane * 16;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    const XT *x = static_cast<const XT *>(a.x), *residual = static_cast<const XT *>(a.residual);
    XT *sum = static_cast<XT *>(a.sum);
    YT *y = static_cast<YT *>(a.y);
    const int64_t step = l.row_step * a.d;                            // elements from one row to the next
    int64_t t = l.row, start = t * a.d - l.shift + l.at, ahead = start;
    int32_t own = (int32_t)l.rows, coming = own;                      // rows to work on, to fetch
    const int32_t turns = SUB < 32 ? (int32_t)__reduce_max_sync(0xffffffffu, (uint32_t)own) : own;       // of the warp's rows together
    auto get = [&](int slot) {
        if (coming > 0) {
            const uint32_t to = ring_at + slot * R::kBytes;
            fetch(to, x, ahead, l);
            if (residual) fetch(to + R::kX, residual, ahead, l);
            --coming;
            ahead += step;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < NP; ++i)
        if (l.mask[i] == 0)
            for (int k = 0; k < R::kStages * 2; ++k)                  // the piece in each stage's two tensors
                for (int h = 0; h < (int)sizeof(XT) / 2; ++h)
                    *reinterpret_cast<uint4 *>(ring + k * R::kX + (i * ((int)sizeof(XT) / 2) + h) * 512) = make_uint4(0, 0, 0, 0);
    for (int k = 0; k < R::kStages - 1; ++k) get(k);
    stage_vector(reinterpret_cast<float *>(smem), a.gamma, 1.0f, a.d, l.shift, room);
    stage_vector(reinterpret_cast<float *>(smem) + room, a.beta, 0.0f, a.d, l.shift, room);
    __syncthreads();
    int32_t mine = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) mine += __popc(l.mask[i]);
    const float n_warp = SUB < 32 ? (float)a.d : (float)__reduce_add_sync(0xffffffffu, mine), share = n_warp > 0.0f ? 1.0f / n_warp : 0.0f, inv_d = 1.0f / (float)a.d;
    int turn = 0, slot = 0;
    for (int32_t k = 0; k < turns; ++k, turn ^= 1, t += l.row_step, start += step) {
        const bool here = SUB == 32 || k < own;
        asm volatile("cp.async.wait_group %0;" :: "n"(R::kStages - 2) : "memory");
        const char *from = ring + slot * R::kBytes;
        Pair v[NP][4], s = both(0.0f);
#pragma unroll
        for (int i = 0; i < NP; ++i) take<XT>(from, i, l, v[i]);
        if (residual) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                Pair r[4];
                take<XT>(from + R::kX, i, l, r);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i][e] = add(v[i][e], r[e]);
                round8<XT>(v[i]);
                if (here) put(sum, start, i, l, v[i]);
            }
        }
        get(slot == 0 ? R::kStages - 1 : slot - 1);                   // into the slot that was taken a row ago
        slot = slot + 1 == R::kStages ? 0 : slot + 1;
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) s = add(s, v[i][e]);
        const float2 s2 = split(s);
        // The sum over n, what it leaves over included (the remainder is exact): times a rounded 1 / n alone, the mean of equal values is often
        // the float next to them, and what is left of them meets a large rstd.  A division takes 2 us more (65536 x 256 bf16: 29.4, 27 so).
        const float total = warp_sum<SUB>(s2.x + s2.y), about = total * share, rest = fmaf(-about, n_warp, total);
        float n = n_warp, mean = fabsf(about) <= 3.4028235e38f ? fmaf(rest, share, about) : about;
        const float local = mean;
        Pair q2 = both(0.0f);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][e] = add(v[i][e], both(-local));
            if (!EVEN && (l.edges >> i & 1u)) Signs(l.mask[i]).keep(v[i]);
            if (l.mask[i] != 0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) q2 = fma2(v[i][e], v[i][e], q2);
            }
        }
        const float2 qq = split(q2);
        float q = warp_sum<SUB>(qq.x + qq.y);
        if (SUB == 32 && sh.warps > 1) {
            const float3 *all = part[turn] + l.group * sh.warps;
            if (l.lane == 0) part[turn][threadIdx.x >> 5] = make_float3(n, mean, q);
            group_sync(l.group, l.threads);
            n = all[0].x; mean = all[0].y; q = all[0].z;
            for (int w = 1; w < sh.warps; ++w) {
                const float3 b = all[w];
                if (b.x > 0.0f) {
                    const float sum_n = n + b.x, delta = b.y - mean, part_b = __fdividef(b.x, sum_n);
                    mean = fmaf(delta, part_b, mean);
                    q += fmaf(delta * delta, n * part_b, b.z);
                    n = sum_n;
                }
            }
        }
        const float rstd = rsqrtf(q * inv_d + a.eps);
        if (l.first && here) {
            if (a.mean) a.mean[t] = mean;
            if (a.rstd) a.rstd[t] = rstd;
        }
        const Pair back = both(local - mean), r2 = both(rstd);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            Pair w[4], b[4];
            read8(gamma + i * 256, w);
            read8(beta + i * 256, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][e] = fma2(mul(add(v[i][e], back), r2), w[e], b[e]);
            if (here) put(y, start, i, l, v[i]);
        }
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

// A thread block walks over rows with a stride; a lane keeps its columns' share of dgamma and dbeta in registers to the end.  8192 x 2048 bf16
// with dsum: 28 us (4.8 TB/s; 33 with the last sums), half of the instruction slots used: a row's two sums are a chain of shuffles and a meeting of four
// warps, which sixteen warps on an SM hide only in part.
template <typename XT, typename YT, int NP, bool EVEN, int SUB>
__global__ void __launch_bounds__(kThreads, NP == 4 ? 1 : 2)
backward_kernel(const BackwardArgs a, const Shape sh, float *__restrict__ partial)
{
    typedef BackwardRing<XT, YT, NP> R;
    __shared__ float2 part[2][kMaxWarps];
    extern __shared__ __align__(16) char smem[];
    pdl_launch_dependents();
    pdl_wait();
    const Lane<NP, EVEN, SUB> l(a.T, a.d, sh.warps, sh.groups, sh.classes);
    const int32_t room = SUB < 32 ? SUB * 8 : sh.warps * NP * 256;
    const float *gamma = reinterpret_cast<const float *>(smem) + l.at;
    char *rings = smem + room * 4, *ring = rings + (threadIdx.x >> 5) * (R::kStages * R::kBytes) + l.lane * 16;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    const XT *x = static_cast<const XT *>(a.x), *dsum = static_cast<const XT *>(a.dsum);
    const YT *dy = static_cast<const YT *>(a.dy);
    XT *dx = static_cast<XT *>(a.dx);
    const int64_t step = l.row_step * a.d;
    int64_t start = l.row * a.d - l.shift + l.at, ahead = start;
    const int32_t own = (int32_t)l.rows, turns = SUB < 32 ? (int32_t)__reduce_max_sync(0xffffffffu, (uint32_t)own) : own;
    int32_t coming = own;
    auto get = [&](int slot) {
        if (coming > 0) {
            const uint32_t to = ring_at + slot * R::kBytes;
            fetch(to, x, ahead, l);
            fetch(to + R::kX, dy, ahead, l);
            if (dsum) fetch(to + R::kX + R::kY, dsum, ahead, l);
            --coming;
            ahead += step;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < NP; ++i)
        if (l.mask[i] == 0)
            for (int k = 0; k < R::kStages; ++k)
                for (int h = 0; h < 2; ++h) {                         // the piece's halves in x, dsum and dy
                    const uint4 zero = make_uint4(0, 0, 0, 0);
                    if (h < (int)sizeof(XT) / 2) {
                        const int at = k * R::kBytes + (i * ((int)sizeof(XT) / 2) + h) * 512;
                        *reinterpret_cast<uint4 *>(ring + at) = *reinterpret_cast<uint4 *>(ring + at + R::kX + R::kY) = zero;
                    }
                    if (h < (int)sizeof(YT) / 2) *reinterpret_cast<uint4 *>(ring + k * R::kBytes + R::kX + (i * ((int)sizeof(YT) / 2) + h) * 512) = zero;
                }
    for (int k = 0; k < R::kStages - 1; ++k) get(k);
    stage_vector(reinterpret_cast<float *>(smem), a.gamma, 1.0f, a.d, l.shift, room);
    __syncthreads();
    Pair dg[NP][4], db[NP][4];
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) dg[i][e] = db[i][e] = both(0.0f);
    const float inv_d = 1.0f / (float)a.d;
    const float *mean = a.mean + l.row, *rstd = a.rstd + l.row;
    float mu_next = 0.0f, rs_next = 0.0f;
    if (own > 0) { mu_next = *mean; rs_next = *rstd; }
    int turn = 0, slot = 0;
    for (int32_t k = 0; k < turns; ++k, turn ^= 1, start += step) {
        const bool here = SUB == 32 || k < own;
        const Pair mu = both(-mu_next), rs = both(rs_next);
        if (k + 1 < own) { mean += l.row_step; rstd += l.row_step; mu_next = *mean; rs_next = *rstd; }
        else if (SUB < 32) mu_next = rs_next = 0.0f;                  // behind the last row h is to be 0: the one before may have an infinite one
        asm volatile("cp.async.wait_group %0;" :: "n"(R::kStages - 2) : "memory");
        const char *from = ring + slot * R::kBytes;
        Pair g[NP][4], h[NP][4], s1 = both(0.0f), s2 = both(0.0f);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            Pair w[4];
            take<XT>(from, i, l, h[i]);
            take<YT>(from + R::kX, i, l, g[i]);
            if (!here) {                                              // the warp's other rows have one more
#pragma unroll
                for (int e = 0; e < 4; ++e) h[i][e] = g[i][e] = both(0.0f);
            }
            read8(gamma + i * 256, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                h[i][e] = mul(add(h[i][e], mu), rs);                  // of a column that the row does not have: meets a g of zero
                db[i][e] = add(db[i][e], g[i][e]);
                dg[i][e] = fma2(g[i][e], h[i][e], dg[i][e]);
                g[i][e] = mul(g[i][e], w[e]);
                s1 = add(s1, g[i][e]);
                s2 = fma2(g[i][e], h[i][e], s2);
            }
        }
        const float2 p1 = split(s1), p2 = split(s2);
        float t1 = p1.x + p1.y, t2 = p2.x + p2.y;
        if (!(fabsf(t2) <= 3.4028235e38f)) {                          // where -mean rstd is beyond all floats, columns that the row lacks gave NaN
            Pair only = both(0.0f);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                Pair c[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) c[e] = mul(g[i][e], h[i][e]);
                Signs(l.mask[i]).keep(c);
#pragma unroll
                for (int e = 0; e < 4; ++e) only = add(only, c[e]);
            }
            const float2 p = split(only);
            t2 = p.x + p.y;
        }
        t1 = warp_sum<SUB>(t1);
        t2 = warp_sum<SUB>(t2);
        if (SUB == 32 && sh.warps > 1) {
            const float2 *all = part[turn] + l.group * sh.warps;
            if (l.lane == 0) part[turn][threadIdx.x >> 5] = make_float2(t1, t2);
            group_sync(l.group, l.threads);
            t1 = t2 = 0.0f;
            for (int w = 0; w < sh.warps; ++w) { t1 += all[w].x; t2 += all[w].y; }
        }
        const Pair m1 = both(-t1 * inv_d), m2 = both(-t2 * inv_d);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            if (dsum) {
                Pair r[4];
                take<XT>(from + R::kX + R::kY, i, l, r);
#pragma unroll
                for (int e = 0; e < 4; ++e) g[i][e] = fma2(fma2(h[i][e], m2, add(g[i][e], m1)), rs, r[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) g[i][e] = mul(fma2(h[i][e], m2, add(g[i][e], m1)), rs);
            }
            if (here) put(dx, start, i, l, g[i]);
        }
        get(slot == 0 ? R::kStages - 1 : slot - 1);                   // into the slot that was taken a row ago
        slot = slot + 1 == R::kStages ? 0 : slot + 1;
    }
    if (!a.dgamma && !a.dbeta) return;
    // the groups' sums, in their order; the rings are done with
    float *columns = reinterpret_cast<float *>(rings);
    float *out_g = gridDim.x == 1 ? a.dgamma : partial + (int64_t)blockIdx.x * 2 * a.d, *out_b = gridDim.x == 1 ? a.dbeta : out_g + a.d;
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float2 *to = reinterpret_cast<float2 *>(columns + l.group * 2 * room + l.at + i * 256 + 2 * e);
            to[0] = split(dg[i][e]);
            to[room / 2] = split(db[i][e]);
        }
    __syncthreads();
    for (int32_t c = threadIdx.x; c < 2 * a.d; c += blockDim.x) {
        const int32_t which = c >= a.d, at = which * room + l.shift + c - which * a.d;
        float t = columns[at];
        for (int k = 1; k < sh.groups; ++k) t += columns[k * 2 * room + at];
        float *out = which ? out_b : out_g;
        if (out) out[c - which * a.d] = t;
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

// Adds the thread blocks' sums in a fixed order: 32 columns to a block, 32 rows of them at a time.
__global__ void __launch_bounds__(1024)
finish_kernel(const float *__restrict__ partial, int32_t parts, int32_t d, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    __shared__ float red[32][33];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, row = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;                // of dgamma's d and dbeta's d
    float t = 0.0f;
    if (c < 2 * (int64_t)d) {
#pragma unroll 10
        for (int32_t k = row; k < parts; k += 32) t += partial[(int64_t)k * 2 * d + c];
    }
    red[lane][row] = t;
    __syncthreads();
    t = warp_sum(red[row][lane]);                                     // warp `row` has column `row` now
    const int64_t o = (int64_t)blockIdx.x * 32 + row;
    if (lane == 0 && o < 2 * (int64_t)d) {
        if (o < d) { if (dgamma) dgamma[o] = t; }
        else if (dbeta) dbeta[o - d] = t;
    }
}

// `most`: pieces to a lane at most, from which on more warps share a row.  The fewest warps of those that leave the fewest lanes without
// columns; four pieces in any case where eight warps need them.
Shape shape_of(int32_t d, int most)
{
    Shape s;
    s.classes = d % 8 == 0 ? 1 : d % 4 == 0 ? 2 : d % 2 == 0 ? 4 : 8;
    const int32_t pieces = (d + 8 - 8 / s.classes + 7) / 8;           // that a row can touch: it begins up to 0, 4, 6 or 7 columns inside of one
    s.lng = pieces > kMaxWarps * 32 * 4;
    s.np = 4; s.warps = kMaxWarps;
    int32_t least = 0x7fffffff;
    for (int np = 1; np <= 4; ++np) {
        const int32_t warps = (pieces + 32 * np - 1) / (32 * np);
        if (warps > kMaxWarps || (np > most && least != 0x7fffffff)) continue;
        if (warps * np < least || (warps * np == least && warps < s.warps)) { least = warps * np; s.np = np; s.warps = (int)warps; }
    }
    s.sub = pieces <= 4 ? 4 : pieces <= 8 ? 8 : pieces <= 16 ? 16 : 32;
    s.groups = s.sub < 32 ? kThreads / s.sub : kMaxWarps / s.warps;
    return s;
}
int threads_of(const Shape &s) { return s.sub < 32 ? kThreads : s.groups * s.warps * 32; }
size_t room_of(const Shape &s) { return (size_t)(s.sub < 32 ? s.sub * 8 : s.warps * s.np * 256) * 4; }        // of a row's columns as floats
constexpr int kMostForward = 4, kMostBackward = 3;
// Thread blocks: two to an SM, and no more than there are rows; as many of each class.
int64_t blocks_of(int64_t T, const Shape &s, int per_sm)
{
    const int64_t most = (int64_t)sm_count() * per_sm / s.classes, need = ((T + s.classes - 1) / s.classes + s.groups - 1) / s.groups;
    return (need < most ? need : most) * s.classes;
}
// The backward pass of a few rows is one thread block's, which writes the columns' sums itself: up to four rows of a group after one another
// take less than a second kernel (the call of 16 x 512: 3.8 us against 5.7).
bool one_block(int64_t T, const Shape &s) { return !s.lng && s.classes == 1 && T <= 4 * s.groups; }
// Dynamic shared memory with which two thread blocks fit on an SM (228 KB, 1 KB of each block's is the system's).
constexpr size_t kHalf = 113 * 1024;
constexpr int kLongParts = 64;

// Early, where the thread blocks fill the GPU or are a handful; those in between would be placed two to an SM while others are empty.
// Forward and backward in a graph, us, early / ordinary: 16 x 512 7.5 / 8.1, 300 x 2048 15.8 / 14.7, 777 x 501 13.3 / 12.3, 1500 x 512
// 12.5 / 11.9; 300 x 501 10.8 / 11.1 goes the other way; from 64 to 8192 rows of other widths the two are within 3 %.
template <typename... KArgs, typename... Args>
cudaError_t launch(int64_t blocks, int per_sm, void (*kernel)(KArgs...), int threads, size_t smem, cudaStream_t s, Args... args)
{
    const dim3 grid((unsigned)blocks), block(threads);
    if (blocks <= 8 || blocks + 8 >= (int64_t)sm_count() * per_sm) return launch_pdl(kernel, grid, block, smem, s, args...);
    return launch_spread(kernel, grid, block, smem, s, args...);
}

template <int I> using Int = std::integral_constant<int, I>;
template <typename E, typename F> cudaError_t with_pieces(const Shape &s, E even, F f)
{
    if (s.sub < 32) return s.sub == 4 ? f(Int<1>{}, even, Int<4>{}) : s.sub == 8 ? f(Int<1>{}, even, Int<8>{}) : f(Int<1>{}, even, Int<16>{});
    return s.np == 1 ? f(Int<1>{}, even, Int<32>{}) : s.np == 2 ? f(Int<2>{}, even, Int<32>{}) : s.np == 3 ? f(Int<3>{}, even, Int<32>{})
                                                                                                       : f(Int<4>{}, even, Int<32>{});
}
template <typename F> cudaError_t with_shape(const Shape &s, F f)
{
    return s.classes == 1 ? with_pieces(s, std::true_type{}, f) : with_pieces(s, std::false_type{}, f);
}

template <typename XT, typename YT> cudaError_t forward_typed(const ForwardArgs &a, cudaStream_t s)
{
    const Shape sh = shape_of(a.d, kMostForward);
    if (sh.lng) {
        const int64_t most = (int64_t)sm_count() * 8;
        return launch_pdl(forward_long_kernel<XT, YT>, dim3((unsigned)(a.T < most ? a.T : most)), dim3(kThreads), 0, s, static_cast<const XT *>(a.x),
                          static_cast<const XT *>(a.residual), a.T, a.d, a.gamma, a.beta, a.eps, static_cast<XT *>(a.sum), static_cast<YT *>(a.y), a.mean,
                          a.rstd);
    }
    return with_shape(sh, [&](auto np, auto even, auto sub) {
        constexpr int NP = decltype(np)::value;
        constexpr bool EVEN = decltype(even)::value;
        constexpr int SUB = decltype(sub)::value;
        typedef ForwardRing<XT, YT, NP> R;
        const size_t smem = 2 * room_of(sh) + (size_t)threads_of(sh) / 32 * R::kStages * R::kBytes;
        static std::atomic<uint64_t> done;
        const cudaError_t e = allow_smem(forward_kernel<XT, YT, NP, EVEN, SUB>, done);
        if (e != cudaSuccess) return e;
        const int per_sm = smem <= kHalf ? 2 : 1;
        return launch(blocks_of(a.T, sh, per_sm), per_sm, forward_kernel<XT, YT, NP, EVEN, SUB>, threads_of(sh), smem, s, a, sh);
    });
}

template <typename XT, typename YT> cudaError_t backward_typed(const BackwardArgs &a, float *partial, cudaStream_t s)
{
    const Shape sh = shape_of(a.d, kMostBackward);
    const bool sums = a.dgamma || a.dbeta;
    int32_t parts = 0;
    cudaError_t e;
    if (sh.lng) {
        const YT *dy = static_cast<const YT *>(a.dy);
        const XT *x = static_cast<const XT *>(a.x);
        const int64_t most = (int64_t)sm_count() * 8;
        e = launch_pdl(backward_long_kernel<XT, YT>, dim3((unsigned)(a.T < most ? a.T : most)), dim3(kThreads), 0, s, dy, x, a.T, a.d, a.gamma,
                       a.mean, a.rstd, static_cast<const XT *>(a.dsum), static_cast<XT *>(a.dx));
        parts = (int32_t)(a.T < kLongParts ? a.T : kLongParts);
        const int32_t slabs = (a.d + kThreads - 1) / kThreads;
        if (e == cudaSuccess && sums)
            e = launch_pdl(column_sums_kernel<XT, YT>, dim3(slabs < 4096 ? slabs : 4096, parts), dim3(kThreads), 0, s, dy, x, a.T, a.d, a.mean,
                           a.rstd, partial);
    } else {
        e = with_shape(sh, [&](auto np, auto even, auto sub) {
            constexpr int NP = decltype(np)::value;
        constexpr bool EVEN = decltype(even)::value;
        constexpr int SUB = decltype(sub)::value;
            typedef BackwardRing<XT, YT, NP> R;
            const size_t room = room_of(sh), rings = (size_t)threads_of(sh) / 32 * R::kStages * R::kBytes;
            const size_t sums_room = (size_t)sh.groups * 2 * room;    // the same space as the rings, which are larger
            const size_t smem = room + (rings > sums_room ? rings : sums_room);
            static std::atomic<uint64_t> done;
            const cudaError_t e1 = allow_smem(backward_kernel<XT, YT, NP, EVEN, SUB>, done);
            if (e1 != cudaSuccess) return e1;
            const int per_sm = NP < 4 && smem <= kHalf ? 2 : 1;
            parts = one_block(a.T, sh) ? 1 : (int32_t)blocks_of(a.T, sh, per_sm);
            return launch(parts, per_sm, backward_kernel<XT, YT, NP, EVEN, SUB>, threads_of(sh), smem, s, a, sh, partial);
        });
    }
    if (e != cudaSuccess || !sums || (!sh.lng && parts == 1)) return e;            // one thread block has written them
    return launch_pdl(finish_kernel, dim3((unsigned)((2 * (int64_t)a.d + 31) / 32)), dim3(1024), 0, s, static_cast<const float *>(partial), parts,
                      a.d, a.dgamma, a.dbeta);
}

}  // namespace

size_t backward_workspace_bytes(int64_t T, int32_t d)
{
    const Shape sh = shape_of(d, kMostBackward);
    if (one_block(T, sh)) return 0;
    const int64_t parts = sh.lng ? (T < kLongParts ? T : kLongParts) : blocks_of(T, sh, 2);        // at most
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
