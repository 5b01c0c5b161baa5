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
#include <type_traits>

#include "adamw.cuh"
#include "vec8.cuh"

namespace tbn {
namespace adamw {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
// Thread blocks to an SM.  With 8-bit states a warp loads its next block while it computes, for which the registers are needed; with 32-bit
// ones there is little to compute and a fourth thread block hides more.
constexpr int step_per_sm(bool eight) { return eight ? 3 : 4; }
constexpr int kNormPerSm = 6, kUnpackPerSm = 8;

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
// A chunk is what a thread block takes at a time: `per` blocks of 256 elements to each warp, so that what a tensor takes to be found and
// set up is paid once for them; one block where there is too little work for every SM otherwise.
template <typename D, int N> struct TableOf {
    D t[N];
    int32_t count, per;
    int64_t chunks;
};
template <int N> using Table = TableOf<Desc, N>;
constexpr int kFew = 24, kMany = 256;       // 2 KB and 22 KB of parameters

template <typename D, int N> __device__ __forceinline__ const D &find(const TableOf<D, N> &tab, int64_t chunk)
{
    int lo = 0, hi = tab.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.t[mid].chunk0 <= chunk) lo = mid; else hi = mid - 1;
    }
    return tab.t[lo];
}

struct Coef {
    float b1, omb1, b2, omb2, eps, step_size, inv_sqrt_bc2;
    float nought;                           // -0
    double lr;
    float gs;
    uint32_t key;
};

// A published 32-bit integer hash of two multiplications: C. Wellons, "Prospecting for Hash Functions" (2018), its variant of least bias.
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x)
{
    x ^= x >> 16; x *= 0x7feb352du;
    x ^= x >> 15; x *= 0x846ca68bu;
    return x ^ (x >> 16);
}

__host__ __device__ inline void set_coef(Coef &c, double lr, double beta1, double beta2, int64_t step, uint64_t seed)
{
    if (step < 1) step = 1;                                           // for the random numbers too
    const double t = (double)step;
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

// A product that an addition follows is written as a b + z with z a -0 that the compiler cannot see through: it joins a packed product
// and the sum that takes it to one rounding, .rn or not, and codes follow from the roundings.
__device__ __forceinline__ Pair product(Pair a, Pair b, Pair z) { return fma2(a, b, z); }
__device__ __forceinline__ Pair add_rz(Pair a, Pair b)
{
    Pair d;
    asm("add.rz.f32x2 %0, %1, %2;" : "=l"(d.r) : "l"(a.r), "l"(b.r));
    return d;
}

__device__ __forceinline__ Pair minus(Pair a, Pair b) { return fma2(b, both(-1.0f), a); }       // one rounding, as a - b
__device__ __forceinline__ Pair minus_square(Pair y, Pair c) { return fma2(mul(c, both(-1.0f)), c, y); }    // y - c c, c c being exact

__device__ __forceinline__ float one_if_less(float a, float b)
{
    float r;
    asm("set.lt.f32.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c)  // NaN if one of them is
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// The codes of y in units of their scale: the largest c with c^2 (c^4) <= y, or the next one, with the probability that makes y
// the mean: where u times the gap is below what y has over c's value.  The floor of an approximate root can be one off where y is within
// 2^-21 of a code's value; the draw then gives that code all the same but for one in 2^16 of them.  Neither passes the largest code: y
// is at most 2^-24 over the top's value, less than the smallest draw asks for.  root: of y (of c^2's size), to be floored.
__device__ __forceinline__ Pair code2(Pair y, Pair root, Pair u)
{
    const Pair c = add(add_rz(root, both(kMagic)), both(-kMagic));
    const Pair over = minus_square(y, c), t = mul(u, fma2(c, both(2.0f), both(1.0f)));
    const float2 o = split(over), d = split(t);
    return add(c, pair(one_if_less(d.x, o.x), one_if_less(d.y, o.y)));
}
__device__ __forceinline__ Pair code4(Pair y, Pair root, Pair u, Pair z)
{
    const Pair c = add(add_rz(root, both(kMagic)), both(-kMagic)), c1 = add(c, both(1.0f));
    const Pair s = mul(c, c), s1 = mul(c1, c1), low = product(s, s, z), next = product(s1, s1, z);
    const Pair over = minus(y, low), t = mul(u, minus(next, low));
    const float2 o = split(over), d = split(t);
    return add(c, pair(one_if_less(d.x, o.x), one_if_less(d.y, o.y)));
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
__device__ __forceinline__ uint32_t bits_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t bits_of(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }
template <bool VEC, typename T> __device__ __forceinline__ void load_raw(const T *p, int cnt, Raw8<T> &r)
{
    if (VEC) { r = load8(p); return; }
    constexpr int kPer = 4 / (int)sizeof(T);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = 32 * e < cnt ? bits_of(p[32 * e]) : 0u;
        if (e % kPer == 0) r.w[e / kPer] = b;
        else r.w[e / kPer] |= b << 16;
    }
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
template <typename PT, typename GT> struct Loaded<PT, GT, false> { Raw8<PT> p; Raw8<GT> g; Raw8<float> m, v; };
template <typename PT, typename GT> struct Loaded<PT, GT, true> { Raw8<PT> p; Raw8<GT> g; uint32_t mc[2], vc[2]; float ms, vs; };

// Where a lane's elements of a block are (VEC: eight in a row, otherwise every 32nd).
template <typename PT, typename GT, bool VEC, bool EIGHT> struct Cursor {
    typedef typename std::conditional<EIGHT, uint8_t, float>::type ST;
    PT *p;
    const GT *g;
    ST *m, *v;
    __nv_bfloat16 *copy;
    float *ms, *vs;
    __device__ __forceinline__ Cursor(const Desc &d, int64_t base)
    {
        const int64_t at = base + (threadIdx.x & 31) * (VEC ? 8 : 1);
        p = static_cast<PT *>(d.p) + at; g = static_cast<const GT *>(d.g) + at;
        m = static_cast<ST *>(d.m) + at; v = static_cast<ST *>(d.v) + at;
        copy = d.copy ? static_cast<__nv_bfloat16 *>(d.copy) + at : nullptr;
        if (EIGHT) { ms = d.ms + base / kBlock; vs = d.vs + base / kBlock; }
    }
    __device__ __forceinline__ void on()
    {
        p += kBlock; g += kBlock; m += kBlock; v += kBlock;
        if (copy) copy += kBlock;
    }
    __device__ __forceinline__ void load(Loaded<PT, GT, EIGHT> &l, int cnt) const
    {
        load_raw<VEC>(p, cnt, l.p);
        load_raw<VEC>(g, cnt, l.g);
        if constexpr (EIGHT) {
            load_codes(m, VEC, cnt, l.mc);
            load_codes(v, VEC, cnt, l.vc);
            l.ms = *ms; l.vs = *vs;
        } else {
            load_raw<VEC>(m, cnt, l.m);
            load_raw<VEC>(v, cnt, l.v);
        }
    }
    __device__ __forceinline__ void store_param(const float (&x)[8], int cnt) const
    {
        store_some(p, VEC, cnt, x);
        if (copy) store_some(copy, VEC, cnt, x);
    }
};

// Blocks on their way from memory: a ring of a warp's own in shared memory, filled by asynchronous copies, so that two blocks are being
// fetched while a third is computed without a register held for them.
constexpr int kStages = 3;
template <typename PT, typename GT> struct Ring {
    static constexpr int kP = 0, kG = kBlock * (int)sizeof(PT), kM = kG + kBlock * (int)sizeof(GT), kV = kM + kBlock, kBytes = kV + kBlock;
    static __device__ __forceinline__ void copy16(uint32_t to, const void *from)
    {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
    }
    static __device__ __forceinline__ void fetch(uint32_t to, const Cursor<PT, GT, true, true> &at, int ahead)
    {
        const int lane = threadIdx.x & 31;
        const int k = ahead * kBlock;
        // 512 bytes to a copy of the warp: of fp32 values the lane's own eight are copied by two lanes
        const char *p = reinterpret_cast<const char *>(at.p + k) - lane * (8 * (int)sizeof(PT) - 16);
        const char *g = reinterpret_cast<const char *>(at.g + k) - lane * (8 * (int)sizeof(GT) - 16);
#pragma unroll
        for (int i = 0; i < (int)sizeof(PT) / 2; ++i) copy16(to + kP + i * 512 + lane * 16, p + i * 512);
#pragma unroll
        for (int i = 0; i < (int)sizeof(GT) / 2; ++i) copy16(to + kG + i * 512 + lane * 16, g + i * 512);
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" :: "r"(to + kM + lane * 8), "l"(at.m + k) : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" :: "r"(to + kV + lane * 8), "l"(at.v + k) : "memory");
    }
    template <typename T> static __device__ __forceinline__ void take8(const char *from, Raw8<T> &r)
    {
        const uint4 *q = reinterpret_cast<const uint4 *>(from + (threadIdx.x & 31) * (8 * sizeof(T)));
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) { const uint4 x = q[i]; r.w[4 * i] = x.x; r.w[4 * i + 1] = x.y; r.w[4 * i + 2] = x.z; r.w[4 * i + 3] = x.w; }
    }
    static __device__ __forceinline__ void take(const char *from, Loaded<PT, GT, true> &l)
    {
        const int lane = threadIdx.x & 31;
        take8(from + kP, l.p);
        take8(from + kG, l.g);
        const uint2 m = *reinterpret_cast<const uint2 *>(from + kM + lane * 8), v = *reinterpret_cast<const uint2 *>(from + kV + lane * 8);
        l.mc[0] = m.x; l.mc[1] = m.y; l.vc[0] = v.x; l.vc[1] = v.y;
    }
};

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

// With 32-bit states.
template <typename PT, typename GT, bool VEC>
__device__ __forceinline__ void step_block(const Cursor<PT, GT, VEC, false> &at, int cnt, const Coef &c, float decay, const Loaded<PT, GT, false> &l)
{
    float p[8], g[8], m[8], v[8];
    unpack8(l.p, p);
    unpack8(l.g, g);
    unpack8(l.m, m);
    unpack8(l.v, v);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        Pair pp = pair(p[e], p[e + 1]), mm = pair(m[e], m[e + 1]), vv = pair(v[e], v[e + 1]);
        float2 root;
        update(c, decay, pair(g[e], g[e + 1]), pp, mm, vv, root);
        f32x2_unpack(pp.r, p[e], p[e + 1]); f32x2_unpack(mm.r, m[e], m[e + 1]); f32x2_unpack(vv.r, v[e], v[e + 1]);
    }
    at.store_param(p, cnt);
    store_some(at.m, VEC, cnt, m);
    store_some(at.v, VEC, cnt, v);
}

// With 8-bit states; the block's new scales go to ms and vs.  k: what the random numbers of the block follow from (the tensor's key and the lane's first element).
template <typename PT, typename GT, bool VEC>
__device__ __forceinline__ void step_block(const Cursor<PT, GT, VEC, true> &at, int cnt, const Coef &c, float decay, uint32_t k,
                                           const Loaded<PT, GT, true> &l, float &ms, float &vs)
{
    float p[8], g[8];
    unpack8(l.p, p);
    unpack8(l.g, g);
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
        m[i] = mul(pair(__fmul_rn(f.x, fabsf(f.x)), __fmul_rn(f.y, fabsf(f.y))), both(l.ms));
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
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        Pair pp = pair(p[2 * i], p[2 * i + 1]);
        update(c, decay, pair(g[2 * i], g[2 * i + 1]), pp, m[i], v[i], root[i]);
        f32x2_unpack(pp.r, p[2 * i], p[2 * i + 1]);
        const float2 fm = split(m[i]), fv = split(v[i]);
        mt = max3_nan(mt, fabsf(fm.x), fabsf(fm.y));
        vt = max3_nan(vt, fv.x, fv.y);
    }
    at.store_param(p, cnt);
    // bits of floats above zero keep their order; those of infinity and NaN come last
    uint32_t mb = __reduce_max_sync(0xffffffffu, __float_as_uint(mt)), vb = __reduce_max_sync(0xffffffffu, __float_as_uint(vt));
    const bool bad = mb >= 0x7f800000u || vb >= 0x7f800000u;
    if (bad) {                                                        // the largest finite magnitudes
        mb = vb = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 fm = split(m[i]), fv = split(v[i]);
            const uint32_t x[4] = {__float_as_uint(fabsf(fm.x)), __float_as_uint(fabsf(fm.y)), __float_as_uint(fv.x), __float_as_uint(fv.y)};
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (x[j] < 0x7f800000u && x[j] > mb) mb = x[j];
                if (x[2 + j] < 0x7f800000u && x[2 + j] > vb) vb = x[2 + j];
            }
        }
        mb = __reduce_max_sync(0xffffffffu, mb);
        vb = __reduce_max_sync(0xffffffffu, vb);
    }
    const float m_top = fmaxf(__uint_as_float(mb), kMLeast), v_top = fmaxf(__uint_as_float(vb), kVLeast);
    const float m_inv = __fdiv_rn(kMTop, m_top), v_inv = __fdiv_rn(kVTop, v_top), v_root = sqrt_fast(v_inv);
    const Pair z = both(c.nought);
    float cm[8], cv[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float hm[2], hv[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // mix(key ^ element): the element is the lane's first one ^ e or 32 e, so the first step of the mix is the lane's; the halves as
            // the low bits of 128 + h / 2^16
            const int e = 2 * i + j;
            uint32_t x = (k ^ (uint32_t)(VEC ? e : 32 * e)) * 0x7feb352du;
            x = (x ^ (x >> 15)) * 0x846ca68bu;
            const uint32_t hi = __byte_perm(x, 0x43000000u, 0x7632);
            hv[j] = __uint_as_float(hi);
            hm[j] = __uint_as_float(hi ^ (x & 0xffffu));
        }
        const Pair shift = both(-(128.0f - 0x1p-17f));                // (h + 1/2) / 2^16, in no order of roundings: it is exact
        const float2 fm = split(m[i]);
        const Pair ym = pair(__fmul_rn(fabsf(fm.x), m_inv), __fmul_rn(fabsf(fm.y), m_inv)), yv = product(v[i], both(v_inv), z);
        const float2 y = split(ym), rv = split(mul(pair(root[i].x, root[i].y), both(v_root)));
        const float2 a = split(code2(ym, pair(sqrt_fast(y.x), sqrt_fast(y.y)), add(pair(hm[0], hm[1]), shift)));
        const Pair b = code4(yv, pair(sqrt_fast(rv.x), sqrt_fast(rv.y)), add(pair(hv[0], hv[1]), shift), z);
        const Pair sm = add(pair(copysignf(a.x, fm.x), copysignf(a.y, fm.y)), both(kMagicSigned)), sv = add(b, both(kMagic));
        f32x2_unpack(sm.r, cm[2 * i], cm[2 * i + 1]);
        f32x2_unpack(sv.r, cv[2 * i], cv[2 * i + 1]);
    }
    uint32_t mc[2] = {low_bytes(cm[0], cm[1], cm[2], cm[3]), low_bytes(cm[4], cm[5], cm[6], cm[7])};
    uint32_t vc[2] = {low_bytes(cv[0], cv[1], cv[2], cv[3]), low_bytes(cv[4], cv[5], cv[6], cv[7])};
    if (bad || has_byte(vc[0], 0) || has_byte(vc[1], 0)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 fm = split(m[e >> 1]), fv = split(v[e >> 1]);
            const float x = e & 1 ? fv.y : fv.x;
            const uint32_t byte = 255u << (8 * (e & 3));
            if (x > 0.0f && (vc[e >> 2] & byte) == 0) vc[e >> 2] |= 0x01010101u & byte;
            if (!(fabsf(e & 1 ? fm.y : fm.x) <= 3.4028235e38f)) mc[e >> 2] = (mc[e >> 2] & ~byte) | (0x80808080u & byte);
            if (!(x <= 3.4028235e38f)) vc[e >> 2] |= byte;
        }
    }
    store_codes(at.m, VEC, cnt, mc);
    store_codes(at.v, VEC, cnt, vc);
    ms = __fmul_rn(m_top, kMPart);
    vs = __fmul_rn(v_top, kVPart);
}

// One step of the tensors of one kind.  32-bit states: HBM; 134 M elements with a bf16 copy take 657 us (6.1 TB/s).  8-bit states: HBM and the
// rate at which instructions issue (66 for an element); 201 M elements with fp32 parameters and bf16 gradients take 546 us (5.2 TB/s; reads
// and writes alone 514 in this order), 20.6 M with bf16 parameters 67.  A warp has its blocks in a row: their scales are whole sectors, where
// scales written one by one cost 60 us more at 201 M, and memory is gone through in long stretches (blocks dealt out in turn: 602 us).
template <int N, typename PT, typename GT, bool EIGHT>
__global__ void __launch_bounds__(kThreads, step_per_sm(EIGHT))
step_kernel(const __grid_constant__ Table<N> tab, const __grid_constant__ Coef host, const __grid_constant__ Hyper h)
{
    __shared__ Coef shared;
    extern __shared__ __align__(16) char rings[];
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
    if (!(fabsf(c.gs) <= 3.4028235e38f)) return;                      // a gradient that is not finite: no step
    for (int64_t chunk = blockIdx.x; chunk < tab.chunks; chunk += gridDim.x) {
        const Desc &d = find(tab, chunk);
        int64_t base = ((chunk - d.chunk0) * kWarps + (threadIdx.x >> 5)) * tab.per * kBlock;
        if (base >= d.n) continue;
        const float decay = (float)(1.0 - c.lr * (double)d.wd);
        // whole blocks of an aligned tensor that the warp has here, then the others
        const int64_t there = d.vec ? (d.n - base) / kBlock : 0;
        int left = tab.per, fast = (int)(there < left ? there : left);
        uint32_t key = 0;
        if (EIGHT) key = mix(c.key + (uint32_t)d.ordinal) ^ mix((uint32_t)(base >> 32));           // a chunk never crosses a multiple of 2^32
        if (fast > 0) {
            Cursor<PT, GT, true, EIGHT> at(d, base);
            if constexpr (EIGHT) {
                typedef Ring<PT, GT> R;
                char *ring = rings + (threadIdx.x >> 5) * (kStages * R::kBytes);
                const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
                auto fetch = [&](int i, int ahead, int slot) {        // one group of copies for each block, empty behind the last one
                    if (i < fast) R::fetch(ring_at + slot * R::kBytes, at, ahead);
                    asm volatile("cp.async.commit_group;" ::: "memory");
                };
                __syncwarp();                                         // the ring's last blocks have been taken
#pragma unroll
                for (int i = 0; i < kStages - 1; ++i) fetch(i, i, i);
                // block i's scales are lane i's
                const int lane = threadIdx.x & 31;
                float ms = 0.0f, vs = 0.0f;
                if (lane < fast) { ms = at.ms[lane]; vs = at.vs[lane]; }
                int slot = 0;
#pragma unroll 1
                for (int i = 0; i < fast; ++i) {
                    asm volatile("cp.async.wait_group %0;" :: "n"(kStages - 2) : "memory");
                    __syncwarp();
                    Loaded<PT, GT, EIGHT> l;
                    R::take(ring + slot * R::kBytes, l);
                    l.ms = __shfl_sync(0xffffffffu, ms, i); l.vs = __shfl_sync(0xffffffffu, vs, i);
                    // into the slot that every lane took before the barrier above
                    fetch(i + kStages - 1, kStages - 1, slot == 0 ? kStages - 1 : slot - 1);
                    slot = slot + 1 == kStages ? 0 : slot + 1;
                    uint32_t k = key ^ ((uint32_t)base + lane * 8);
                    float m_new, v_new;
                    step_block(at, 256, c, decay, k ^ (k >> 16), l, m_new, v_new);
                    if (lane == i) { ms = m_new; vs = v_new; }
                    base += kBlock;
                    at.on();
                }
                if (lane < fast) { at.ms[lane] = ms; at.vs[lane] = vs; }
            } else {
#pragma unroll 1
                for (int i = 0; i < fast; ++i, at.on(), base += kBlock) {
                    Loaded<PT, GT, EIGHT> l;
                    at.load(l, 256);
                    step_block(at, 256, c, decay, l);
                }
            }
            left -= fast;
        }
#pragma unroll 1
        for (; left > 0 && base < d.n; --left, base += kBlock) {
            const Cursor<PT, GT, false, EIGHT> at(d, base);
            const int64_t rest = d.n - base - (threadIdx.x & 31);
            const int cnt = (int)(rest < 256 ? rest : 256);           // elements at 32 e < cnt exist
            Loaded<PT, GT, EIGHT> l;
            at.load(l, cnt);
            if constexpr (EIGHT) {
                uint32_t k = key ^ ((uint32_t)base + (threadIdx.x & 31));
                float ms, vs;
                step_block(at, cnt, c, decay, k ^ (k >> 16), l, ms, vs);
                if ((threadIdx.x & 31) == 0) { *at.ms = ms; *at.vs = vs; }
            } else {
                step_block(at, cnt, c, decay, l);
            }
        }
    }
}

// ---- values of 8-bit states ---------------------------------------------------------------------------------------------
// Two bytes read and eight written an element: 355 us for 201 M (5.7 TB/s), what a stream of mostly writes reaches.
struct UnpackDesc {
    const uint8_t *m, *v;
    const float *ms, *vs;
    float *m_out, *v_out;
    int64_t n, chunk0;
    int32_t vec;
};
template <int N> using UnpackTable = TableOf<UnpackDesc, N>;

template <int N>
__global__ void __launch_bounds__(kThreads)
unpack_kernel(const __grid_constant__ UnpackTable<N> tab)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    for (int64_t chunk = blockIdx.x; chunk < tab.chunks; chunk += gridDim.x) {
        const UnpackDesc &d = find(tab, chunk);
        int64_t base = ((chunk - d.chunk0) * tab.per * kWarps + (threadIdx.x >> 5)) * kBlock;
        for (int i = 0; i < tab.per && base < d.n; ++i, base += kWarps * kBlock) {
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
}

// ---- global norm of the gradients ---------------------------------------------------------------------------------------
struct NormDesc {
    const void *g;
    int64_t n, chunk0;
    int32_t bf16, vec;
};
template <int N> using NormTable = TableOf<NormDesc, N>;

// Squares are added in 64 bits from the first one on: the factor that the norm gives enters every element of a step, and sums of 32 bits
// would be off in its last bits.  |g| is made a 64-bit number by shifts of its bits (201 M bf16 gradients: 70 us; with the conversion
// instruction 144, with pairs of fp32 sums 100).  Zero and subnormal numbers become 2^-127 to 2^-126 that way: the last kernel takes a
// sum below 2^-200 for 0.  Infinities and NaN become 2^128 and more: a thread whose sum is 2^256 goes over its elements again with the
// conversion.
__device__ __forceinline__ void add_squares(const Raw8<float> &r, double (&sums)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t a = r.w[e] & 0x7fffffffu;
        const double x = __hiloint2double((int)((a >> 3) + (896u << 20)), (int)(a << 29));
        sums[e] = fma(x, x, sums[e]);
    }
}
__device__ __forceinline__ void add_squares(const Raw8<__nv_bfloat16> &r, double (&sums)[8])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const double lo = __hiloint2double((int)((r.w[e] & 0x7fffu) * 8192u + (896u << 20)), 0);
        const double hi = __hiloint2double((int)(((r.w[e] & 0x7fff0000u) >> 3) + (896u << 20)), 0);
        sums[2 * e] = fma(lo, lo, sums[2 * e]);
        sums[2 * e + 1] = fma(hi, hi, sums[2 * e + 1]);
    }
}

template <int N>
__global__ void __launch_bounds__(kThreads)
norm_kernel(const __grid_constant__ NormTable<N> tab, double *__restrict__ partial)
{
    __shared__ double warp_sum[kWarps];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    constexpr int kStride = kWarps * kBlock;
    // f(what a lane has of a block, as loaded)
    auto go_over = [&](auto f) {
        auto tensor = [&](const auto *g, const NormDesc &d, int64_t base) {
            typedef typename std::remove_cv<typename std::remove_reference<decltype(*g)>::type>::type GT;
            constexpr int kGroup = 8 / (int)sizeof(GT);
            int left = tab.per;
            // whole blocks of an aligned tensor in groups, one group loaded while the one before it is added up
            const int64_t there = d.vec && d.n - base >= kBlock ? (d.n - base - kBlock) / kStride + 1 : 0;
            const int count = (int)(there < left ? there : left) / kGroup;
            if (count > 0) {
                Raw8<GT> r[kGroup], ahead[kGroup];
                const GT *at = g + base + lane * 8;
#pragma unroll
                for (int i = 0; i < kGroup; ++i) r[i] = load8(at + i * kStride);
#pragma unroll 1
                for (int k = 1;; ++k) {
                    at += kGroup * kStride;
                    if (k < count) {
#pragma unroll
                        for (int i = 0; i < kGroup; ++i) ahead[i] = load8(at + i * kStride);
                    }
#pragma unroll
                    for (int i = 0; i < kGroup; ++i) f(r[i]);
                    if (k >= count) break;
#pragma unroll
                    for (int i = 0; i < kGroup; ++i) r[i] = ahead[i];
                }
                left -= count * kGroup;
                base += (int64_t)count * kGroup * kStride;
            }
#pragma unroll 1
            for (; left > 0 && base < d.n; --left, base += kStride) {
                const int64_t rest = d.n - base;
                Raw8<GT> r;
                if (d.vec && rest >= kBlock) load_raw<true>(g + base + lane * 8, 256, r);
                else load_raw<false>(g + base + lane, (int)(rest - lane < 256 ? rest - lane : 256), r);
                f(r);
            }
        };
        for (int64_t chunk = blockIdx.x; chunk < tab.chunks; chunk += gridDim.x) {
            const NormDesc &d = find(tab, chunk);
            const int64_t base = ((chunk - d.chunk0) * tab.per * kWarps + (threadIdx.x >> 5)) * kBlock;
            if (d.bf16) tensor(static_cast<const __nv_bfloat16 *>(d.g), d, base);
            else tensor(static_cast<const float *>(d.g), d, base);
        }
    };
    double sums[8] = {};
    go_over([&](const auto &r) { add_squares(r, sums); });
    double sum = ((sums[0] + sums[1]) + (sums[2] + sums[3])) + ((sums[4] + sums[5]) + (sums[6] + sums[7]));
    if (sum >= 0x1p256) {
        sum = 0.0;
        go_over([&](const auto &r) {
            float g[8];
            unpack8(r, g);
#pragma unroll 1
            for (int e = 0; e < 8; ++e) sum = fma((double)g[e], (double)g[e], sum);
        });
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    if (lane == 0) warp_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) t += warp_sum[w];
        partial[blockIdx.x] = t;
    }
}

// One block adds the thread blocks' sums, in an order that their number decides.
__global__ void __launch_bounds__(1024)
norm_final_kernel(const double *__restrict__ partial, int32_t count, double max_norm, float *__restrict__ norm, float *__restrict__ scale)
{
    __shared__ double red[32];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double t = 0.0;
    for (int32_t i = threadIdx.x; i < count; i += 1024) t += partial[i];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
    if (lane == 0) red[warp] = t;
    __syncthreads();
    if (warp != 0) return;
    t = red[lane];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
    if (lane == 0) {
        const double len = t < 0x1p-200 ? 0.0 : sqrt(t);
        if (norm) *norm = (float)len;
        const bool finite = len <= 1.7976931348623157e308;
        if (scale) *scale = !finite ? __int_as_float(0x7fffffff) : len > max_norm ? (float)(max_norm / len) : 1.0f;
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------
bool at8(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) % (size_t)(8 * bytes)) == 0; }
unsigned grid_of(int64_t chunks, int per_sm)
{
    const int64_t most = (int64_t)sm_count() * per_sm;
    return (unsigned)(chunks < most ? chunks : most);
}

// Runs `put` and `go` over the tensors that `want` picks, as many to a launch as a table holds.
template <typename D, typename Put, typename Go, typename Want>
int in_tables(const tbn_adamw_tensor *tensors, int32_t count, int per_sm, int least_per, int most_per, Want want, Put put, Go go)
{
    int32_t picked = 0;
    for (int32_t i = 0; i < count; ++i) picked += tensors[i].n > 0 && want(tensors[i]);
    int32_t i = 0;
    while (picked > 0) {
        auto fill = [&](auto &tab, int most) {
            int64_t blocks = 0;
            for (tab.count = 0; i < count && tab.count < most; ++i) {
                if (tensors[i].n <= 0 || !want(tensors[i])) continue;
                auto &d = tab.t[tab.count++];
                put(d, tensors[i], i);
                d.n = tensors[i].n;
                blocks += (d.n + kBlock - 1) / kBlock;
            }
            picked -= tab.count;
            // as many blocks to a warp as leave the thread blocks two chunks each
            const int64_t round = (int64_t)sm_count() * per_sm * kWarps;
            tab.per = least_per;
            while (tab.per < most_per && blocks >= 4 * round * tab.per) tab.per *= 2;
            const int64_t chunk = (int64_t)tab.per * kWarps * kBlock;
            tab.chunks = 0;
            for (int32_t k = 0; k < tab.count; ++k) {
                tab.t[k].chunk0 = tab.chunks;
                tab.chunks += (tab.t[k].n + chunk - 1) / chunk;
            }
        };
        int rc;
        if (picked <= kFew) { TableOf<D, kFew> tab; fill(tab, kFew); rc = go(tab, std::integral_constant<int, kFew>{}); }
        else { TableOf<D, kMany> tab; fill(tab, kMany); rc = go(tab, std::integral_constant<int, kMany>{}); }
        if (rc != TBN_OK) return rc;
    }
    return TBN_OK;
}

template <typename PT, typename GT, bool EIGHT>
int step_kind(const tbn_adamw_tensor *tensors, int32_t count, const Hyper &h, const Coef &host, cudaStream_t s)
{
    const int pd = sizeof(PT) == 2 ? TBN_BF16 : TBN_F32, gd = sizeof(GT) == 2 ? TBN_BF16 : TBN_F32;
    return in_tables<Desc>(
        tensors, count, step_per_sm(EIGHT), 1, EIGHT ? 8 : 4,
        [&](const tbn_adamw_tensor &t) { return t.param_dtype == pd && t.grad_dtype == gd && (t.state_bits == 8) == EIGHT; },
        [&](Desc &d, const tbn_adamw_tensor &t, int32_t i) {
            d.p = t.param; d.g = t.grad; d.m = t.m; d.v = t.v; d.ms = t.m_scale; d.vs = t.v_scale; d.copy = t.copy;
            d.wd = t.weight_decay; d.ordinal = i;
            const int sb = EIGHT ? 1 : 4;
            d.vec = at8(t.param, sizeof(PT)) && at8(t.grad, sizeof(GT)) && at8(t.m, sb) && at8(t.v, sb) && (!t.copy || at8(t.copy, 2));
        },
        [&](const auto &tab, auto size) {
            auto kernel = step_kernel<decltype(size)::value, PT, GT, EIGHT>;
            const int smem = EIGHT ? kWarps * kStages * Ring<PT, GT>::kBytes : 0;
            static std::atomic<uint64_t> done;
            if (smem > 0 && allow_smem(kernel, done) != cudaSuccess) return (int)TBN_ERR_CUDA;
            return launch_pdl(kernel, dim3(grid_of(tab.chunks, step_per_sm(EIGHT))), dim3(kThreads), smem, s, tab, host, h) == cudaSuccess
                       ? (int)TBN_OK : (int)TBN_ERR_CUDA;
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
    return in_tables<UnpackDesc>(
        tensors, count, kUnpackPerSm, 1, 4, [](const tbn_adamw_tensor &) { return true; },
        [&](UnpackDesc &d, const tbn_adamw_tensor &t, int32_t i) {
            d.m = static_cast<const uint8_t *>(t.m); d.v = static_cast<const uint8_t *>(t.v);
            d.ms = t.m_scale; d.vs = t.v_scale;
            d.m_out = m ? m[i] : nullptr; d.v_out = v ? v[i] : nullptr;
            d.vec = at8(t.m, 1) && at8(t.v, 1) && at8(d.m_out, 4) && at8(d.v_out, 4);
        },
        [&](const auto &tab, auto size) {
            return launch_pdl(unpack_kernel<decltype(size)::value>, dim3(grid_of(tab.chunks, kUnpackPerSm)), dim3(kThreads), 0, s, tab) ==
                           cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
        });
}

size_t norm_workspace_bytes(int32_t count)
{
    return (size_t)(count / kMany + 1) * sm_count() * kNormPerSm * sizeof(double);
}

int launch_norm(const tbn_adamw_tensor *tensors, int32_t count, double max_norm, float *norm, float *scale, void *workspace, cudaStream_t s)
{
    double *partial = static_cast<double *>(workspace);
    int32_t used = 0;
    int rc = in_tables<NormDesc>(
        tensors, count, kNormPerSm, 4, 16, [](const tbn_adamw_tensor &) { return true; },
        [&](NormDesc &d, const tbn_adamw_tensor &t, int32_t) {
            d.g = t.grad; d.bf16 = t.grad_dtype == TBN_BF16; d.vec = at8(t.grad, d.bf16 ? 2 : 4);
        },
        [&](const auto &tab, auto size) {
            const unsigned grid = grid_of(tab.chunks, kNormPerSm);
            double *out = partial + used;
            used += (int32_t)grid;
            return launch_pdl(norm_kernel<decltype(size)::value>, dim3(grid), dim3(kThreads), 0, s, tab, out) == cudaSuccess
                       ? TBN_OK : TBN_ERR_CUDA;
        });
    if (rc != TBN_OK) return rc;
    return launch_pdl(norm_final_kernel, dim3(1), dim3(1024), 0, s, static_cast<const double *>(partial), used, max_norm, norm, scale) ==
                   cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
}

}  // namespace adamw
}  // namespace tbn
