// Eight consecutive fp32 or bf16 values of a lane: one 32-byte or 16-byte access (a warp's request covers whole lines).
#pragma once

#include <atomic>

#include "common.cuh"

namespace tbn {

template <typename T> struct Raw8;                                   // as loaded: fp32 and bf16 keep their bits until they are used
template <> struct Raw8<float> { uint32_t w[8]; };
template <> struct Raw8<__nv_bfloat16> { uint32_t w[4]; };

__device__ __forceinline__ Raw8<float> load8(const float *p)
{
    Raw8<float> r;
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
                 : "l"(p) : "memory");
    return r;
}
__device__ __forceinline__ Raw8<__nv_bfloat16> load8(const __nv_bfloat16 *p)
{
    Raw8<__nv_bfloat16> r;
    asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(p) : "memory");
    return r;
}
__device__ __forceinline__ void unpack8(const Raw8<float> &r, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(r.w[e]);
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16> &r, float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(r.w[e] << 16);
        v[2 * e + 1] = __uint_as_float(r.w[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])),
                    "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])) : "memory");
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&v)[8])
{
    asm volatile("st.global.v4.b32 [%0], {%1,%2,%3,%4};"
                 :: "l"(p), "r"(pack_bf16(v[0], v[1])), "r"(pack_bf16(v[2], v[3])), "r"(pack_bf16(v[4], v[5])), "r"(pack_bf16(v[6], v[7]))
                 : "memory");
}

// Two fp32 values to an instruction, where the rate at which instructions issue is what bounds a kernel.  (The compiler may join a
// product and the sum that takes it to one rounding.)
struct Pair { uint64_t r; };
__device__ __forceinline__ Pair pair(float a, float b) { return {f32x2_pack(a, b)}; }
__device__ __forceinline__ Pair both(float a) { return pair(a, a); }
__device__ __forceinline__ float2 split(Pair p) { float2 f; f32x2_unpack(p.r, f.x, f.y); return f; }
__device__ __forceinline__ Pair mul(Pair a, Pair b) { return {f32x2_mul(a.r, b.r)}; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { return {f32x2_fma(a.r, b.r, c.r)}; }
__device__ __forceinline__ Pair add(Pair a, Pair b)
{
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.r) : "l"(a.r), "l"(b.r));
    return d;
}
// Raw8 as four pairs, and back.
__device__ __forceinline__ void unpack8(const Raw8<float> &r, Pair (&v)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pair(__uint_as_float(r.w[2 * e]), __uint_as_float(r.w[2 * e + 1]));
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16> &r, Pair (&v)[4])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pair(__uint_as_float(r.w[e] << 16), __uint_as_float(r.w[e] & 0xffff0000u));
}
__device__ __forceinline__ void spread8(const Pair (&v)[4], float (&f)[8])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) f32x2_unpack(v[e].r, f[2 * e], f[2 * e + 1]);
}

// Lets a kernel have the largest dynamic shared memory, once for each device.  `done`: the kernel's own, one bit for a device.
template <typename K> cudaError_t allow_smem(K kernel, std::atomic<uint64_t> &done)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = (uint64_t)1 << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    cudaFuncAttributes at;
    e = cudaFuncGetAttributes(&at, kernel);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - (int)at.sharedSizeBytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}
// An ordinary launch, for the first kernel of a call where it has few small blocks that are to lie on SMs of their own: launched early
// (launch_pdl) they are placed while the kernel before holds most SMs, several on each of the few that are free.
template <typename... KArgs, typename... Args>
cudaError_t launch_spread(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = s;
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}
// Multiprocessors of the current device.
inline int sm_count()
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

__device__ __forceinline__ float value_of(float v) { return v; }
__device__ __forceinline__ float value_of(__nv_bfloat16 v) { return __bfloat162float(v); }

}  // namespace tbn
