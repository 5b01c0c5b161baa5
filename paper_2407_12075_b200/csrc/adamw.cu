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
    float nought;                           // -0
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
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float rcp_fast(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

constexpr float kMTop = 127.0f * 127.0f, kVTop = 254.0f * 254.0f * 254.0f * 254.0f;
constexpr float kMPart = (float)(1.0 / (127.0 * 127.0)), kVPart = (float)(1.0 / (254.0 * 254.0 * 254.0 * 254.0));
constexpr float kMLeast = 0x1p-100f, kVLeast = 0x1p-94f;
constexpr float kMagic = 8388608.0f, kMagicSigned = 12582912.0f;     // 2^23, 1.5 2^23: an integer added to one of them is in its low bits

// Two fp32 values to an instruction: the arithmetic of 8-bit states is bound by the rate at which instructions issue.
struct Pair { uint64_t r; };
__device__ __forceinline__ Pair pair(float a, float b) { return {f32x2_pack(a, b)}; }
__device__ __forceinline__ Pair both(float a) { return pair(a, a); }
__device__ __forceinline__ float2 split(Pair p) { float2 f; f32x2_unpack(p.r, f.x, f.y); return f; }
__device__ __forceinline__ Pair mul(Pair a, Pair b) { return {f32x2_mul(a.r, b.r)}; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { return {f32x2_fma(a.r, b.r, c.r)}; }
// A product that an addition follows is written as a b + z with z a -0 that the compiler cannot see through: it joins a packed product
// and the sum that takes it to one rounding, .rn or not, and codes follow from the roundings.
__device__ __forceinline__ Pair product(Pair a, Pair b, Pair z) { return fma2(a, b, z); }
__device__ __forceinline__ Pair add(Pair a, Pair b)
{
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.r) : "l"(a.r), "l"(b.r));
    return d;
}
__device__ __forceinline__ Pair add_rz(Pair a, Pair b)
{
    Pair d;
    asm("add.rz.f32x2 %0, %1, %2;" : "=l"(d.r) : "l"(a.r), "l"(b.r));
    return d;
}

__device__ __forceinline__ Pair minus(Pair a, Pair b) { return fma2(b, both(-1.0f), a); }       // one rounding, as a - b
__device__ __forceinline__ Pair minus_square(Pair y, Pair c) { return fma2(mul(c, both(-1.0f)), c, y); }    // y - c c, c c being exact

// The codes of y in units of their scale: the largest c with c^2 (c^4) <= y, or the next one, with the probability that makes y
// the mean: where (h + 1/2) / 2^16 times the gap is below what y has over c's value.  The floor of an approximate root can be
// one off where y is within 2^-21 of a code's value; the draw then gives that code all the same but for one in 2^16 of them.
// Neither passes the largest code: y is at most 2^-24 over the top's value, less than the smallest draw asks for.
// hm, hv: the random halves, as 2^23 + h.  root: of y (of c^2's size), to be floored.
__device__ __forceinline__ Pair code2(Pair y, Pair root, Pair hm)
{
    const Pair c = add(add_rz(root, both(kMagic)), both(-kMagic));
    const Pair over = minus_square(y, c);
    const Pair t = mul(add(hm, both(-8388607.5f)), fma2(c, both(2.0f), both(1.0f)));
    const float2 o = split(mul(over, both(65536.0f))), d = split(t), f = split(c);
    return pair(d.x < o.x ? f.x + 1.0f : f.x, d.y < o.y ? f.y + 1.0f : f.y);
}
__device__ __forceinline__ Pair code4(Pair y, Pair root, Pair hv, Pair z)
{
    const Pair c = add(add_rz(root, both(kMagic)), both(-kMagic)), c1 = add(c, both(1.0f));
    const Pair s = mul(c, c), s1 = mul(c1, c1), low = product(s, s, z), next = product(s1, s1, z);
    const Pair t = mul(add(hv, both(-8388607.5f)), minus(next, low));
    const float2 o = split(mul(minus(y, low), both(65536.0f))), d = split(t), f = split(c);
    return pair(d.x < o.x ? f.x + 1.0f : f.x, d.y < o.y ? f.y + 1.0f : f.y);
}

__device__ __forceinline__ float m_value(int32_t c, float ms)
{
    const float f = (float)c;
    return c == -128 ? __int_as_float(0x7fffffff) : __fmul_rn(__fmul_rn(f, fabsf(f)), ms);
}
__device__ __forceinline__ float v_value(uint32_t c, float vs)
{
    const float f = (float)c, s = __fmul_rn(f, f);
    return c == 255u ? __int_as_float(0x7f800000) : __fmul_rn(__fmul_rn(s, s), vs);
}
__device__ __forceinline__ bool has_byte(uint32_t w, uint32_t four)     // one of w's bytes is that of `four`, whose bytes are all the same
{
    const uint32_t x = w ^ four;
    return ((x - 0x01010101u) & ~x & 0x80808080u) != 0;
}
__device__ __forceinline__ uint32_t low_bytes(float a, float b, float c, float d)
{
    const uint32_t lo = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), hi = __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
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

// What a lane holds of a block, as loaded.
template <typename PT, typename GT, bool EIGHT> struct Loaded;
template <typename PT, typename GT> struct Loaded<PT, GT, false> { float p[8], g[8], m[8], v[8]; };
template <typename PT, typename GT> struct Loaded<PT, GT, true> { float p[8], g[8]; uint32_t mc[2], vc[2]; float ms, vs; };

// Where a lane's elements are: the first one, and elements at 32 e < cnt exist.
template <bool VEC> struct Place {
    int64_t at;
    int cnt;
    __device__ __forceinline__ Place(const Desc &d, int64_t base)
    {
        const int lane = threadIdx.x & 31;
        const int64_t left = d.n - base - lane;
        at = base + (VEC ? lane * 8 : lane);
        cnt = VEC ? 256 : (int)(left < 256 ? left : 256);
    }
};

template <typename PT, typename GT, bool VEC, bool EIGHT>
__device__ __forceinline__ void load_block(const Desc &d, int64_t base, Loaded<PT, GT, EIGHT> &l)
{
    const Place<VEC> w(d, base);
    load_some(static_cast<const PT *>(d.p) + w.at, VEC, w.cnt, l.p);
    load_some(static_cast<const GT *>(d.g) + w.at, VEC, w.cnt, l.g);
    if constexpr (EIGHT) {
        load_codes(static_cast<const uint8_t *>(d.m) + w.at, VEC, w.cnt, l.mc);
        load_codes(static_cast<const uint8_t *>(d.v) + w.at, VEC, w.cnt, l.vc);
        l.ms = d.ms[base / kBlock]; l.vs = d.vs[base / kBlock];
    } else {
        load_some(static_cast<const float *>(d.m) + w.at, VEC, w.cnt, l.m);
        load_some(static_cast<const float *>(d.v) + w.at, VEC, w.cnt, l.v);
    }
}

// m, v and the parameter of two elements; the order of the roundings is the documented formula's.
__device__ __forceinline__ void update(const Coef &c, float decay, Pair g, Pair &p, Pair &m, Pair &v, float2 &root)
{
    g = mul(g, both(c.gs));
    const Pair z = both(c.nought);
    m = add(product(m, both(c.b1), z), product(g, both(c.omb1), z));
    v = add(product(v, both(c.b2), z), product(mul(g, both(c.omb2)), g, z));
    const float2 vv = split(v);
    root = make_float2(sqrt_fast(vv.x), sqrt_fast(vv.y));
    const float2 denom = split(fma2(pair(root.x, root.y), both(c.inv_sqrt_bc2), both(c.eps)));
    const Pair step = mul(m, both(-c.step_size));
    p = fma2(step, pair(rcp_fast(denom.x), rcp_fast(denom.y)), mul(p, both(decay)));
}

template <typename PT, typename GT, bool VEC, bool EIGHT>
__device__ __forceinline__ void step_block(const Desc &d, int64_t base, const Coef &c, float decay, uint32_t key, Loaded<PT, GT, EIGHT> &l)
{
    const Place<VEC> w(d, base);
    if constexpr (!EIGHT) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            Pair p = pair(l.p[e], l.p[e + 1]), m = pair(l.m[e], l.m[e + 1]), v = pair(l.v[e], l.v[e + 1]);
            float2 root;
            update(c, decay, pair(l.g[e], l.g[e + 1]), p, m, v, root);
            f32x2_unpack(p.r, l.p[e], l.p[e + 1]); f32x2_unpack(m.r, l.m[e], l.m[e + 1]); f32x2_unpack(v.r, l.v[e], l.v[e + 1]);
        }
        store_some(static_cast<PT *>(d.p) + w.at, VEC, w.cnt, l.p);
        if (d.copy) store_some(static_cast<__nv_bfloat16 *>(d.copy) + w.at, VEC, w.cnt, l.p);
        store_some(static_cast<float *>(d.m) + w.at, VEC, w.cnt, l.m);
        store_some(static_cast<float *>(d.v) + w.at, VEC, w.cnt, l.v);
    } else {
        const int lane = threadIdx.x & 31;
        Pair m[4], v[4];
        float2 root[4];
        const uint32_t mx[2] = {l.mc[0] ^ 0x80808080u, l.mc[1] ^ 0x80808080u};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t wm = mx[i >> 1], wv = l.vc[i >> 1];
            const int b = (2 * i) & 3;
            // the byte as the low bits of 2^23 + code
            const Pair cm = add(pair(__uint_as_float(__byte_perm(wm, 0x4b000000u, 0x7550 + b)), __uint_as_float(__byte_perm(wm, 0x4b000000u, 0x7551 + b))),
                                both(-8388736.0f));
            const Pair cv = add(pair(__uint_as_float(__byte_perm(wv, 0x4b000000u, 0x7550 + b)), __uint_as_float(__byte_perm(wv, 0x4b000000u, 0x7551 + b))),
                                both(-kMagic));
            const float2 f = split(cm);
            m[i] = mul(mul(cm, pair(fabsf(f.x), fabsf(f.y))), both(l.ms));
            const Pair s = mul(cv, cv);
            v[i] = mul(mul(s, s), both(l.vs));
        }
        if (has_byte(l.mc[0], 0x80808080u) || has_byte(l.mc[1], 0x80808080u) || has_byte(l.vc[0], 0xffffffffu) || has_byte(l.vc[1], 0xffffffffu)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t wm = l.mc[i >> 1] >> (16 * (i & 1)), wv = l.vc[i >> 1] >> (16 * (i & 1));
                m[i] = pair(m_value((int32_t)(int8_t)wm, l.ms), m_value((int32_t)(int8_t)(wm >> 8), l.ms));
                v[i] = pair(v_value(wv & 255u, l.vs), v_value((wv >> 8) & 255u, l.vs));
            }
        }
        float mt = 0.0f, vt = 0.0f;
        Pair odd = both(0.0f);                                        // a NaN as soon as there is an infinity or a NaN
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Pair p = pair(l.p[2 * i], l.p[2 * i + 1]);
            update(c, decay, pair(l.g[2 * i], l.g[2 * i + 1]), p, m[i], v[i], root[i]);
            f32x2_unpack(p.r, l.p[2 * i], l.p[2 * i + 1]);
            odd = fma2(m[i], both(0.0f), odd);
            odd = fma2(v[i], both(0.0f), odd);
            const float2 fm = split(m[i]), fv = split(v[i]);
            mt = fmaxf(fmaxf(fabsf(fm.x), fabsf(fm.y)), mt);
            vt = fmaxf(fmaxf(fv.x, fv.y), vt);
        }
        store_some(static_cast<PT *>(d.p) + w.at, VEC, w.cnt, l.p);
        if (d.copy) store_some(static_cast<__nv_bfloat16 *>(d.copy) + w.at, VEC, w.cnt, l.p);
        const float2 oo = split(odd);
        const bool bad = !(oo.x + oo.y == 0.0f);
        if (bad) {                                                    // the largest finite magnitudes
            mt = vt = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 fm = split(m[i]), fv = split(v[i]);
                const float x[4] = {fabsf(fm.x), fabsf(fm.y), fv.x, fv.y};
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (x[k] <= 3.4028235e38f) mt = fmaxf(mt, x[k]);
                    if (x[2 + k] <= 3.4028235e38f) vt = fmaxf(vt, x[2 + k]);
                }
            }
        }
        // bits of floats above zero keep their order
        const float m_top = fmaxf(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(mt))), kMLeast);
        const float v_top = fmaxf(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(vt))), kVLeast);
        const float m_inv = __fdiv_rn(kMTop, m_top), v_inv = __fdiv_rn(kVTop, v_top), v_root = sqrt_fast(v_inv);
        // element e of the lane is w.at ^ (e or 32 e), whose upper half is w.at's: the first step of the mix is the lane's
        uint32_t k = key;
        if (w.at >> 32) k ^= mix((uint32_t)(w.at >> 32));
        k ^= (uint32_t)w.at;
        k ^= k >> 16;
        const Pair z = both(c.nought);
        float cm[8], cv[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float hm[2], hv[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int e = 2 * i + j;
                uint32_t x = (k ^ (uint32_t)(VEC ? e : 32 * e)) * 0x7feb352du;
                x = (x ^ (x >> 15)) * 0x846ca68bu;
                const uint32_t hi = __byte_perm(x, 0x4b000000u, 0x7632);                 // 0x4b00 and the upper half
                hv[j] = __uint_as_float(hi);
                hm[j] = __uint_as_float(hi ^ (x & 0xffffu));
            }
            const float2 fm = split(m[i]), fv = split(v[i]);
            const Pair ym = product(pair(fabsf(fm.x), fabsf(fm.y)), both(m_inv), z), yv = product(v[i], both(v_inv), z);
            const float2 y = split(ym), rv = split(mul(pair(root[i].x, root[i].y), both(v_root)));
            const float2 a = split(code2(ym, pair(sqrt_fast(y.x), sqrt_fast(y.y)), pair(hm[0], hm[1])));
            const float2 b = split(code4(yv, pair(sqrt_fast(rv.x), sqrt_fast(rv.y)), pair(hv[0], hv[1]), z));
            const Pair sm = add(pair(copysignf(a.x, fm.x), copysignf(a.y, fm.y)), both(kMagicSigned));
            const Pair sv = add(pair(fmaxf(b.x, fv.x > 0.0f ? 1.0f : 0.0f), fmaxf(b.y, fv.y > 0.0f ? 1.0f : 0.0f)), both(kMagic));
            f32x2_unpack(sm.r, cm[2 * i], cm[2 * i + 1]);
            f32x2_unpack(sv.r, cv[2 * i], cv[2 * i + 1]);
        }
        uint32_t mc[2] = {low_bytes(cm[0], cm[1], cm[2], cm[3]), low_bytes(cm[4], cm[5], cm[6], cm[7])};
        uint32_t vc[2] = {low_bytes(cv[0], cv[1], cv[2], cv[3]), low_bytes(cv[4], cv[5], cv[6], cv[7])};
        if (bad) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 fm = split(m[e >> 1]), fv = split(v[e >> 1]);
                const uint32_t byte = 255u << (8 * (e & 3));
                if (!(fabsf(e & 1 ? fm.y : fm.x) <= 3.4028235e38f)) mc[e >> 2] = (mc[e >> 2] & ~byte) | (0x80808080u & byte);
                if (!((e & 1 ? fv.y : fv.x) <= 3.4028235e38f)) vc[e >> 2] |= byte;
            }
        }
        store_codes(static_cast<uint8_t *>(d.m) + w.at, VEC, w.cnt, mc);
        store_codes(static_cast<uint8_t *>(d.v) + w.at, VEC, w.cnt, vc);
        if (lane == 0) {
            d.ms[base / kBlock] = __fmul_rn(m_top, kMPart);
            d.vs[base / kBlock] = __fmul_rn(v_top, kVPart);
        }
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
        const float decay = (float)(1.0 - c.lr * (double)d.wd);
        const uint32_t key = mix(c.key + (uint32_t)d.ordinal);
        Loaded<PT, GT, EIGHT> l;
        if (d.vec && d.n - base >= kBlock) {
            load_block<PT, GT, true, EIGHT>(d, base, l);
            step_block<PT, GT, true, EIGHT>(d, base, c, decay, key, l);
        } else {
            load_block<PT, GT, false, EIGHT>(d, base, l);
            step_block<PT, GT, false, EIGHT>(d, base, c, decay, key, l);
        }
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
    double sums[8] = {};                                              // a chain of additions each
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
        for (int e = 0; e < 8; ++e) sums[e] = fma((double)g[e], (double)g[e], sums[e]);
    }
    double sum = ((sums[0] + sums[1]) + (sums[2] + sums[3])) + ((sums[4] + sums[5]) + (sums[6] + sums[7]));
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
    c.nought = -0.0f;
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
