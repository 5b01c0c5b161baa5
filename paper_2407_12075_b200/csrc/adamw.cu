// AdamW over many tensors in one launch, with 32-bit or 8-bit states, and what goes with it: the global norm of the gradients and
// the values of 8-bit states.  Every element is read and written once, so HBM bounds all of it: 28 bytes an element with fp32
// parameters, gradients and states.  A warp takes a block of 256 elements of one tensor, eight to a lane.
//
// 8-bit states.  A block has a scale for m and one for v, from its largest magnitudes.  m = c |c| ms with c in -127..127 and
// v = c^4 vs with c in 0..254: the codes' values lie closer together towards zero, 127 : 1 in m's size becomes 16129 : 1, and
// sqrt(v), what the update divides by, spans 64516 : 1.  A v above zero keeps a code above zero, so that no update is divided by
// eps alone.  Code -128 of m is NaN (infinities too: what they give is NaN), code 255 of v infinity.
// Rounding is at random, with the value as its mean: with beta2 = 0.999 a step moves v by a thousandth where the codes are a
// sixtieth apart at best, and rounded to nearest it would stay where it is for good.
#include <atomic>

#include "adamw.cuh"
#include "vec8.cuh"

namespace tbn {
namespace adamw {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = kThreads * 8;        // elements that a thread block takes at a time

struct Desc {
    void *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    void *copy;
    int64_t n;
    int64_t chunk0;                         // chunks of the tensors before this one
    float wd;
    int32_t ordinal;
    int32_t vec;                            // every pointer begins where an access of eight elements may
};

// Tensors go to the kernel in its parameters: nothing to copy, nothing that a captured graph could find changed.
template <int N> struct Table {
    Desc t[N];
    int32_t count;
    int64_t chunks;
};
constexpr int kFew = 24, kMany = 256;       // 2 KB and 22 KB of parameters

template <int N> __device__ __forceinline__ int find(const Table<N> &tab, int64_t chunk)
{
    int lo = 0, hi = tab.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.t[mid].chunk0 <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}

struct Coef {
    float b1, omb1, b2, omb2, eps, step_size, inv_sqrt_bc2;
    double lr;
    float gs;
    uint32_t key;
};

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16; x *= 0x7feb352du;
    x ^= x >> 15; x *= 0x846ca68bu;
    return x ^ (x >> 16);
}

__host__ __device__ inline void set_coef(Coef &c, double lr, double beta1, double beta2, int64_t step, uint64_t seed)
{
    const double t = (double)(step < 1 ? 1 : step);
    c.lr = lr;
    c.step_size = (float)(lr / (1.0 - pow(beta1, t)));
    c.inv_sqrt_bc2 = (float)(1.0 / sqrt(1.0 - pow(beta2, t)));
    c.key = mix(mix((uint32_t)seed) ^ (uint32_t)step) + mix((uint32_t)(seed >> 32)) + mix((uint32_t)((uint64_t)step >> 32));
}

__device__ __forceinline__ float sqrt_fast(float x)
{
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float floor_small(float x) { return __fadd_rz(x, 8388608.0f) - 8388608.0f; }     // 0 <= x < 2^22
__device__ __forceinline__ float unit(uint32_t h16) { return __uint_as_float(0x3f800000u | (h16 << 7)) - (1.0f - 0x1p-17f); }   // (h16 + 1/2) / 2^16

constexpr float kMTop = 127.0f * 127.0f, kVTop = 254.0f * 254.0f * 254.0f * 254.0f;
constexpr float kMPart = (float)(1.0 / (127.0 * 127.0)), kVPart = (float)(1.0 / (254.0 * 254.0 * 254.0 * 254.0));
constexpr float kMLeast = 0x1p-100f, kVLeast = 0x1p-94f;

// The codes of y in units of their scale: the largest c with c^2 (c^4) <= y, or the next one with the probability that makes y
// the mean.  The first guess may be off by one; every comparison is exact or in a stated order of fp32 operations, so a code
// does not depend on how a root is evaluated.
__device__ __forceinline__ float code2(float y, float u)
{
    float c = floor_small(sqrt_fast(y));
    if (__fmul_rn(c, c) > y) c -= 1.0f;
    if (__fmul_rn(c + 1.0f, c + 1.0f) <= y) c += 1.0f;
    const float low = __fmul_rn(c, c), next = __fmul_rn(c + 1.0f, c + 1.0f);
    if (__fmul_rn(u, next - low) < y - low) c += 1.0f;
    return fminf(c, 127.0f);
}
__device__ __forceinline__ float fourth(float c) { const float s = __fmul_rn(c, c); return __fmul_rn(s, s); }
__device__ __forceinline__ float code4(float y, float u)
{
    float c = floor_small(sqrt_fast(sqrt_fast(y)));
    if (fourth(c) > y) c -= 1.0f;
    if (fourth(c + 1.0f) <= y) c += 1.0f;
    const float low = fourth(c), next = fourth(c + 1.0f);
    if (__fmul_rn(u, next - low) < y - low) c += 1.0f;
    return fminf(c, 254.0f);
}

__device__ __forceinline__ float m_value(int32_t c, float ms)
{
    const float f = (float)c;
    return c == -128 ? __int_as_float(0x7fffffff) : __fmul_rn(__fmul_rn(f, fabsf(f)), ms);
}
__device__ __forceinline__ float v_value(uint32_t c, float vs)
{
    return c == 255u ? __int_as_float(0x7f800000) : __fmul_rn(fourth((float)c), vs);
}

// Elements of a lane: first, first + stride, ... (eight in a row where the tensor is aligned, every 32nd otherwise).
template <typename T> __device__ __forceinline__ void load_some(const T *p, bool vec, int cnt, float (&v)[8])
{
    if (vec) { unpack8(load8(p), v); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 32 * e < cnt ? value_of(p[32 * e]) : 0.0f;
}
template <typename T> __device__ __forceinline__ void store_some(T *p, bool vec, int cnt, const float (&v)[8])
{
    if (vec) { store8(p, v); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (32 * e < cnt) store_from_float(p, 32 * e, v[e]);
}
__device__ __forceinline__ void load_codes(const uint8_t *p, bool vec, int cnt, uint32_t (&w)[2])
{
    if (vec) {
        const uint2 t = *reinterpret_cast<const uint2 *>(p);
        w[0] = t.x; w[1] = t.y;
        return;
    }
    w[0] = w[1] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) if (32 * e < cnt) w[e >> 2] |= (uint32_t)p[32 * e] << (8 * (e & 3));
}
__device__ __forceinline__ void store_codes(uint8_t *p, bool vec, int cnt, const uint32_t (&w)[2])
{
    if (vec) { *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]); return; }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (32 * e < cnt) p[32 * e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
}

template <typename PT, typename GT, bool EIGHT>
__device__ __forceinline__ void step_block(const Desc &d, int64_t base, const Coef &c, float decay, uint32_t key)
{
    const int lane = threadIdx.x & 31;
    const int64_t left = d.n - base;                                  // of the tensor, from the block's first element on
    const bool vec = d.vec && left >= kBlock;
    const int64_t at = base + (vec ? lane * 8 : lane);
    const int stride = vec ? 1 : 32;
    const int cnt = vec ? 256 : (int)(left - lane < 256 ? left - lane : 256);      // elements at 32 e < cnt exist
    float p[8], g[8], m[8], v[8];
    load_some(static_cast<const PT *>(d.p) + at, vec, cnt, p);
    load_some(static_cast<const GT *>(d.g) + at, vec, cnt, g);
    if (EIGHT) {
        uint32_t mc[2], vc[2];
        load_codes(static_cast<const uint8_t *>(d.m) + at, vec, cnt, mc);
        load_codes(static_cast<const uint8_t *>(d.v) + at, vec, cnt, vc);
        const float ms = d.ms[base / kBlock], vs = d.vs[base / kBlock];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = m_value((int32_t)(int8_t)(mc[e >> 2] >> (8 * (e & 3))), ms);
            v[e] = v_value((vc[e >> 2] >> (8 * (e & 3))) & 255u, vs);
        }
    } else {
        load_some(static_cast<const float *>(d.m) + at, vec, cnt, m);
        load_some(static_cast<const float *>(d.v) + at, vec, cnt, v);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float gg = __fmul_rn(g[e], c.gs);
        m[e] = __fadd_rn(__fmul_rn(m[e], c.b1), __fmul_rn(gg, c.omb1));
        v[e] = __fadd_rn(__fmul_rn(v[e], c.b2), __fmul_rn(__fmul_rn(gg, c.omb2), gg));
        const float denom = fmaf(sqrt_fast(v[e]), c.inv_sqrt_bc2, c.eps);
        p[e] = __fmul_rn(p[e], decay) - __fdividef(__fmul_rn(m[e], c.step_size), denom);
    }
    store_some(static_cast<PT *>(d.p) + at, vec, cnt, p);
    if (d.copy) store_some(static_cast<__nv_bfloat16 *>(d.copy) + at, vec, cnt, p);
    if (!EIGHT) {
        store_some(static_cast<float *>(d.m) + at, vec, cnt, m);
        store_some(static_cast<float *>(d.v) + at, vec, cnt, v);
        return;
    }
    uint32_t mt = 0, vt = 0;                                          // largest finite magnitudes: bits of floats above zero keep their order
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t a = __float_as_uint(fabsf(m[e])), b = __float_as_uint(v[e]);
        mt = a < 0x7f800000u && a > mt ? a : mt;
        vt = b < 0x7f800000u && b > vt ? b : vt;
    }
    const float m_top = fmaxf(__uint_as_float(__reduce_max_sync(0xffffffffu, mt)), kMLeast);
    const float v_top = fmaxf(__uint_as_float(__reduce_max_sync(0xffffffffu, vt)), kVLeast);
    const float m_inv = __fdiv_rn(kMTop, m_top), v_inv = __fdiv_rn(kVTop, v_top);
    uint32_t mc[2] = {0, 0}, vc[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int64_t j = at + e * stride;
        uint32_t k = key;
        if (j >> 32) k ^= mix((uint32_t)(j >> 32));
        const uint32_t h = mix((uint32_t)j ^ k);
        const float am = fabsf(m[e]);
        uint32_t cm = 0x80u, cv = 0xffu;
        if (am <= 3.4028235e38f) {
            const int32_t q = (int32_t)code2(__fmul_rn(am, m_inv), unit(h & 0xffffu));
            cm = (uint32_t)(m[e] < 0.0f ? -q : q) & 255u;
        }
        if (v[e] <= 3.4028235e38f) {
            const float q = code4(__fmul_rn(v[e], v_inv), unit(h >> 16));
            cv = (uint32_t)(v[e] > 0.0f ? fmaxf(q, 1.0f) : q);
        }
        mc[e >> 2] |= cm << (8 * (e & 3));
        vc[e >> 2] |= cv << (8 * (e & 3));
    }
    store_codes(static_cast<uint8_t *>(d.m) + at, vec, cnt, mc);
    store_codes(static_cast<uint8_t *>(d.v) + at, vec, cnt, vc);
    if (lane == 0) {
        d.ms[base / kBlock] = __fmul_rn(m_top, kMPart);
        d.vs[base / kBlock] = __fmul_rn(v_top, kVPart);
    }
}

template <int N, typename PT, typename GT, bool EIGHT>
__global__ void __launch_bounds__(kThreads)
step_kernel(const __grid_constant__ Table<N> tab, const __grid_constant__ Coef host, const __grid_constant__ Hyper h)
{
    __shared__ Coef shared;
    pdl_launch_dependents();
    pdl_wait();
    if (threadIdx.x == 0) {
        Coef c = host;
        if (h.step_dev || h.lr_dev)
            set_coef(c, h.lr_dev ? (double)*h.lr_dev : h.lr, h.beta1, h.beta2, h.step_dev ? *h.step_dev : h.step, h.seed);
        c.gs = h.grad_scale ? *h.grad_scale : 1.0f;
        shared = c;
    }
    __syncthreads();
    const Coef c = shared;
    if (!(fabsf(c.gs) <= 3.4028235e38f)) return;                      // gradients without a finite norm: no step
    for (int64_t chunk = blockIdx.x; chunk < tab.chunks; chunk += gridDim.x) {
        const Desc &d = tab.t[find(tab, chunk)];
        const int64_t base = (chunk - d.chunk0) * kChunk + (threadIdx.x >> 5) * kBlock;
        if (base >= d.n) continue;
        step_block<PT, GT, EIGHT>(d, base, c, (float)(1.0 - c.lr * (double)d.wd), mix(c.key + (uint32_t)d.ordinal));
    }
}

// ---- values of 8-bit states ---------------------------------------------------------------------------------------------
struct UnpackDesc {
    const uint8_t *m, *v;
    const float *ms, *vs;
    float *m_out, *v_out;
    int64_t n, chunk0;
    int32_t vec;
};
template <int N> struct UnpackTable {
    UnpackDesc t[N];
    int32_t count;
    int64_t chunks;
};

template <int N>
__global__ void __launch_bounds__(kThreads)
unpack_kernel(const __grid_constant__ UnpackTable<N> tab)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    for (int64_t chunk = blockIdx.x; chunk < tab.chunks; chunk += gridDim.x) {
        int lo = 0, hi = tab.count - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (tab.t[mid].chunk0 <= chunk) lo = mid; else hi = mid - 1;
        }
        const UnpackDesc &d = tab.t[lo];
        const int64_t base = (chunk - d.chunk0) * kChunk + (threadIdx.x >> 5) * kBlock;
        if (base >= d.n) continue;
        const int64_t left = d.n - base;
        const bool vec = d.vec && left >= kBlock;
        const int64_t at = base + (vec ? lane * 8 : lane);
        const int cnt = vec ? 256 : (int)(left - lane < 256 ? left - lane : 256);
        uint32_t mc[2], vc[2];
        load_codes(d.m + at, vec, cnt, mc);
        load_codes(d.v + at, vec, cnt, vc);
        const float ms = d.ms[base / kBlock], vs = d.vs[base / kBlock];
        float m[8], v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = m_value((int32_t)(int8_t)(mc[e >> 2] >> (8 * (e & 3))), ms);
            v[e] = v_value((vc[e >> 2] >> (8 * (e & 3))) & 255u, vs);
        }
        if (d.m_out) store_some(d.m_out + at, vec, cnt, m);
        if (d.v_out) store_some(d.v_out + at, vec, cnt, v);
    }
}

// ---- global norm of the gradients ---------------------------------------------------------------------------------------
struct NormDesc {
    const void *g;
    int64_t n, chunk0;
    int32_t bf16, vec;
};
template <int N> struct NormTable {
    NormDesc t[N];
    int32_t count;
    int64_t chunks;
};

// Squares are added in 64 bits from the first one on: nothing overflows, and the order of the sums is fixed by the sizes.
template <int N>
__global__ void __launch_bounds__(kThreads)
norm_kernel(const __grid_constant__ NormTable<N> tab, double *__restrict__ partial)
{
    __shared__ double warp_sum[kThreads / 32];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    double sum = 0.0;
    for (int64_t chunk = blockIdx.x; chunk < tab.chunks; chunk += gridDim.x) {
        int lo = 0, hi = tab.count - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (tab.t[mid].chunk0 <= chunk) lo = mid; else hi = mid - 1;
        }
        const NormDesc &d = tab.t[lo];
        const int64_t base = (chunk - d.chunk0) * kChunk + (threadIdx.x >> 5) * kBlock;
        if (base >= d.n) continue;
        const int64_t left = d.n - base;
        const bool vec = d.vec && left >= kBlock;
        const int64_t at = base + (vec ? lane * 8 : lane);
        const int cnt = vec ? 256 : (int)(left - lane < 256 ? left - lane : 256);
        float g[8];
        if (d.bf16) load_some(static_cast<const __nv_bfloat16 *>(d.g) + at, vec, cnt, g);
        else load_some(static_cast<const float *>(d.g) + at, vec, cnt, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fma((double)g[e], (double)g[e], sum);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    if (lane == 0) warp_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) t += warp_sum[w];
        partial[blockIdx.x] = t;
    }
}

__global__ void __launch_bounds__(kThreads)
norm_final_kernel(const double *__restrict__ partial, int32_t count, double max_norm, float *__restrict__ norm, float *__restrict__ scale)
{
    __shared__ double red[kThreads];
    pdl_launch_dependents();
    pdl_wait();
    double t = 0.0;
    for (int32_t i = threadIdx.x; i < count; i += kThreads) t += partial[i];
    red[threadIdx.x] = t;
    __syncthreads();
    for (int off = kThreads / 2; off > 0; off >>= 1) {
        if ((int)threadIdx.x < off) red[threadIdx.x] += red[threadIdx.x + off];
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        const double len = sqrt(red[0]);
        if (norm) *norm = (float)len;
        const bool finite = len <= 1.7976931348623157e308;
        if (scale) *scale = !finite ? __int_as_float(0x7fffffff) : len > max_norm ? (float)(max_norm / len) : 1.0f;
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
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

bool at8(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) % (size_t)(8 * bytes)) == 0; }
int64_t chunks_of(int64_t n) { return (n + kChunk - 1) / kChunk; }
unsigned grid_of(int64_t chunks, int per_sm)
{
    const int64_t most = (int64_t)sm_count() * per_sm;
    return (unsigned)(chunks < most ? chunks : most);
}

// Runs `put` and `go` over the tensors that `want` picks, as many to a launch as a table holds.
template <template <int> class Tab, typename Put, typename Go, typename Want>
int in_tables(const tbn_adamw_tensor *tensors, int32_t count, Want want, Put put, Go go)
{
    int32_t picked = 0;
    for (int32_t i = 0; i < count; ++i) picked += tensors[i].n > 0 && want(tensors[i]);
    int32_t i = 0;
    while (picked > 0) {
        auto fill = [&](auto &tab, int most) {
            tab.count = 0; tab.chunks = 0;
            for (; i < count && tab.count < most; ++i) {
                if (tensors[i].n <= 0 || !want(tensors[i])) continue;
                auto &d = tab.t[tab.count++];
                put(d, tensors[i], i);
                d.n = tensors[i].n;
                d.chunk0 = tab.chunks;
                tab.chunks += chunks_of(tensors[i].n);
            }
            picked -= tab.count;
        };
        int rc;
        if (picked <= kFew) { Tab<kFew> tab; fill(tab, kFew); rc = go(tab); }
        else { Tab<kMany> tab; fill(tab, kMany); rc = go(tab); }
        if (rc != TBN_OK) return rc;
    }
    return TBN_OK;
}

template <typename PT, typename GT, bool EIGHT>
int step_kind(const tbn_adamw_tensor *tensors, int32_t count, const Hyper &h, const Coef &host, cudaStream_t s)
{
    const int pd = sizeof(PT) == 2 ? TBN_BF16 : TBN_F32, gd = sizeof(GT) == 2 ? TBN_BF16 : TBN_F32;
    return in_tables<Table>(
        tensors, count,
        [&](const tbn_adamw_tensor &t) { return t.param_dtype == pd && t.grad_dtype == gd && (t.state_bits == 8) == EIGHT; },
        [&](Desc &d, const tbn_adamw_tensor &t, int32_t i) {
            d.p = t.param; d.g = t.grad; d.m = t.m; d.v = t.v; d.ms = t.m_scale; d.vs = t.v_scale; d.copy = t.copy;
            d.wd = t.weight_decay; d.ordinal = i;
            const int sb = EIGHT ? 1 : 4;
            d.vec = at8(t.param, sizeof(PT)) && at8(t.grad, sizeof(GT)) && at8(t.m, sb) && at8(t.v, sb) && (!t.copy || at8(t.copy, 2));
        },
        [&](const auto &tab) {
            auto go = [&](auto kernel) {
                return launch_pdl(kernel, dim3(grid_of(tab.chunks, 4)), dim3(kThreads), 0, s, tab, host, h) == cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
            };
            return go(step_kernel<sizeof(tab.t) / sizeof(Desc), PT, GT, EIGHT>);
        });
}

}  // namespace

int launch_step(const tbn_adamw_tensor *tensors, int32_t count, const Hyper &h, cudaStream_t s)
{
    Coef c = {};
    c.b1 = (float)h.beta1; c.omb1 = (float)(1.0 - h.beta1);
    c.b2 = (float)h.beta2; c.omb2 = (float)(1.0 - h.beta2);
    c.eps = (float)h.eps;
    set_coef(c, h.lr, h.beta1, h.beta2, h.step, h.seed);
    int rc = step_kind<float, float, false>(tensors, count, h, c, s);
    if (rc == TBN_OK) rc = step_kind<float, __nv_bfloat16, false>(tensors, count, h, c, s);
    if (rc == TBN_OK) rc = step_kind<__nv_bfloat16, float, false>(tensors, count, h, c, s);
    if (rc == TBN_OK) rc = step_kind<__nv_bfloat16, __nv_bfloat16, false>(tensors, count, h, c, s);
    if (rc == TBN_OK) rc = step_kind<float, float, true>(tensors, count, h, c, s);
    if (rc == TBN_OK) rc = step_kind<float, __nv_bfloat16, true>(tensors, count, h, c, s);
    if (rc == TBN_OK) rc = step_kind<__nv_bfloat16, float, true>(tensors, count, h, c, s);
    if (rc == TBN_OK) rc = step_kind<__nv_bfloat16, __nv_bfloat16, true>(tensors, count, h, c, s);
    return rc;
}

int launch_unpack(const tbn_adamw_tensor *tensors, int32_t count, float *const *m, float *const *v, cudaStream_t s)
{
    return in_tables<UnpackTable>(
        tensors, count, [](const tbn_adamw_tensor &) { return true; },
        [&](UnpackDesc &d, const tbn_adamw_tensor &t, int32_t i) {
            d.m = static_cast<const uint8_t *>(t.m); d.v = static_cast<const uint8_t *>(t.v);
            d.ms = t.m_scale; d.vs = t.v_scale;
            d.m_out = m ? m[i] : nullptr; d.v_out = v ? v[i] : nullptr;
            d.vec = at8(t.m, 1) && at8(t.v, 1) && at8(d.m_out, 4) && at8(d.v_out, 4);
        },
        [&](const auto &tab) {
            return launch_pdl(unpack_kernel<sizeof(tab.t) / sizeof(UnpackDesc)>, dim3(grid_of(tab.chunks, 8)), dim3(kThreads), 0, s, tab) ==
                           cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
        });
}

constexpr int kNormPerSm = 8;

size_t norm_workspace_bytes(int32_t count)
{
    return (size_t)(count / kMany + 1) * sm_count() * kNormPerSm * sizeof(double);
}

int launch_norm(const tbn_adamw_tensor *tensors, int32_t count, double max_norm, float *norm, float *scale, void *workspace, cudaStream_t s)
{
    double *partial = static_cast<double *>(workspace);
    int32_t used = 0;
    int rc = in_tables<NormTable>(
        tensors, count, [](const tbn_adamw_tensor &) { return true; },
        [&](NormDesc &d, const tbn_adamw_tensor &t, int32_t) {
            d.g = t.grad; d.bf16 = t.grad_dtype == TBN_BF16; d.vec = at8(t.grad, d.bf16 ? 2 : 4);
        },
        [&](const auto &tab) {
            const unsigned grid = grid_of(tab.chunks, kNormPerSm);
            double *out = partial + used;
            used += (int32_t)grid;
            return launch_pdl(norm_kernel<sizeof(tab.t) / sizeof(NormDesc)>, dim3(grid), dim3(kThreads), 0, s, tab, out) == cudaSuccess
                       ? TBN_OK : TBN_ERR_CUDA;
        });
    if (rc != TBN_OK) return rc;
    return launch_pdl(norm_final_kernel, dim3(1), dim3(kThreads), 0, s, static_cast<const double *>(partial), used, max_norm, norm, scale) ==
                   cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
}

}  // namespace adamw
}  // namespace tbn
