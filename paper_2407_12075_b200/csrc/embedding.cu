// Embedding lookup with scaling, from a table or from a tiled table's bits, and the table's gradient.
//
//   y_t = scale table[id_t],   dw_v = scale sum_{t: id_t = v} dy_t     (ids outside the vocabulary: y_t = 0, no gradient)
//
// Both are bound by HBM.  The gradient adds rows in the order of the tokens, whatever the GPU does first: the tokens are sorted by id (stable;
// few by counting in one launch, many by digits of the id), equal pieces of the sorted list are summed by a warp each, 256 to 1024 columns
// at a time, and where an id's tokens go on over several pieces the pieces' sums are added in order by a kernel of their own.  No row of
// dy is read twice, no atomic decides an order.  A whole table is filled with zeros by thread blocks of the sorting launches, whose work
// leaves most SMs free.
//
// No kernel here lets its successor be placed before it ends: waiting blocks would take the registers and shared memory of blocks that are
// still to come (16384 x 2048 step over 50021 ids: 106 us with early placement, 92 without).
#include "embedding.cuh"
#include "vec8.cuh"

namespace tbn {
namespace embed {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ bool inside(int64_t id, int32_t V, int64_t padding) { return id >= 0 && id < V && id != padding; }

// Eight values in a row, 16-byte aligned.
__device__ __forceinline__ void load_row(const __nv_bfloat16 *p, Raw8<__nv_bfloat16> &r) { r = load8(p); }
__device__ __forceinline__ void load_row(const float *p, Raw8<float> &r)
{
    const uint4 a = reinterpret_cast<const uint4 *>(p)[0], b = reinterpret_cast<const uint4 *>(p)[1];
    r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w; r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
}
// Eight values in a row from any element on, asked for (ask) and put together (take) apart, so that several are on their way at a time.
// bf16: cut out of the two aligned pieces that hold them, or value by value where the second reaches behind `end`, the tensor's.
template <typename T, bool ALIGNED> struct OddPiece {
    Raw8<T> r;
    __device__ __forceinline__ void ask(const T *p, const T *)
    {
        if (ALIGNED) load_row(p, r);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) r.w[e % (int)(sizeof(r.w) / 4)] = __float_as_uint(value_of(p[e]));     // fp32
    }
    __device__ __forceinline__ Raw8<T> take(const T *, const T *) const { return r; }
};
template <> struct OddPiece<__nv_bfloat16, false> {
    Raw8<__nv_bfloat16> r;
    uint4 second;
    static __device__ __forceinline__ uint32_t off(const __nv_bfloat16 *p) { return (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u) / 2; }
    __device__ __forceinline__ void ask(const __nv_bfloat16 *p, const __nv_bfloat16 *end)
    {
        const __nv_bfloat16 *q = p - off(p), *q2 = q + 16 <= end ? q + 8 : q;
        const uint4 a = *reinterpret_cast<const uint4 *>(q);
        second = *reinterpret_cast<const uint4 *>(q2);
        r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
    }
    __device__ __forceinline__ Raw8<__nv_bfloat16> take(const __nv_bfloat16 *p, const __nv_bfloat16 *end) const
    {
        Raw8<__nv_bfloat16> o;
        const uint32_t k = off(p);
        if (p - k + 16 > end && k != 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) o.w[e] = __bfloat16_as_ushort(p[2 * e]) | (uint32_t)__bfloat16_as_ushort(p[2 * e + 1]) << 16;
            return o;
        }
        const bool two = k & 4, one = k & 2;                          // words to leave out, in two steps: 2, then 1
        const uint32_t v[6] = {two ? r.w[2] : r.w[0], two ? r.w[3] : r.w[1], two ? second.x : r.w[2], two ? second.y : r.w[3],
                               two ? second.z : second.x, two ? second.w : second.y};
        uint32_t x[5];
#pragma unroll
        for (int e = 0; e < 5; ++e) x[e] = one ? v[e + 1] : v[e];
#pragma unroll
        for (int e = 0; e < 4; ++e) o.w[e] = __funnelshift_r(x[e], x[e + 1], k & 1 ? 16 : 0);
        return o;
    }
};
__device__ __forceinline__ void store_row(float *p, const float (&v)[8])          // 16-byte aligned
{
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store_row(__nv_bfloat16 *p, const float (&v)[8]) { store8(p, v); }
// The eight columns from c on of row `row` of a table, scaled; what is behind column d is left as it is in v.
template <typename WT, bool EVEN> struct DenseRows {
    const WT *table, *end;
    int32_t d;
    float scale;
    struct Row { const WT *at; };
    __device__ __forceinline__ Row row(int64_t id) const { return {table + id * d}; }
    typedef OddPiece<WT, EVEN> Piece;
    __device__ __forceinline__ void load(const Row &r, int32_t c, Piece &p) const { p.ask(r.at + c, end); }
    __device__ __forceinline__ void values(const Row &r, int32_t c, const Piece &p, float (&v)[8]) const
    {
        unpack8(p.take(r.at + c, end), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
    }
    __device__ __forceinline__ float one(const Row &r, int32_t c) const { return value_of(r.at[c]) * scale; }
};
// The same from a tiled table: bit (f mod q) and scaling factor (f / q) of element f = id d + c.
struct TiledRows {
    const uint32_t *tile;
    const float *alpha;
    int64_t q, words;                       // words that the tile occupies
    int32_t d, rows;                        // rows of the table that a tile spans, 0 if it ends inside of one
    int per_tile;
    float scale;
    struct Row { int64_t i; int32_t j; };   // the row's first bit and factor
    __device__ __forceinline__ Row row(int64_t id) const
    {
        if (rows > 0) { const int32_t j = (int32_t)id / rows; return {(int64_t)((int32_t)id - j * rows) * d, j}; }
        const int64_t f = id * d, j = f / q;
        return {f - j * q, (int32_t)j};
    }
    struct Piece { uint32_t bits; float a; };
    __device__ __forceinline__ void place(const Row &r, int32_t c, int64_t &i, int64_t &j) const
    {
        i = r.i + c; j = r.j;
        if (i >= q) { const int64_t more = i / q; j += more; i -= more * q; }
    }
    __device__ __forceinline__ void load(const Row &r, int32_t c, Piece &p) const
    {
        int64_t i, j;
        place(r, c, i, j);
        p.a = i + 8 <= q ? __ldg(alpha + (per_tile ? j : 0)) * scale : -1.0f;         // -1: the piece goes over a tile's end
        const int64_t w = i >> 5;
        const uint32_t lo = __ldg(tile + w), hi = (i & 31) > 24 && w + 1 < words ? __ldg(tile + w + 1) : 0;
        p.bits = __funnelshift_r(lo, hi, (uint32_t)(i & 31));
    }
    __device__ __forceinline__ void values(const Row &r, int32_t c, const Piece &p, float (&v)[8]) const
    {
        if (p.a == -1.0f) {
#pragma unroll
            for (int e = 0; e < 8; ++e) if (c + e < d) v[e] = one(r, c + e);
            return;
        }
        const uint32_t a = __float_as_uint(p.a);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(a ^ (~(p.bits << (31 - e)) & 0x80000000u));
    }
    __device__ __forceinline__ float one(const Row &r, int32_t c) const
    {
        int64_t i, j;
        place(r, c, i, j);
        const float a = __ldg(alpha + (per_tile ? j : 0)) * scale;
        return tile_bit(tile, i) ? a : -a;
    }
};

// A warp takes up to 1024 columns of one token, which it loads before it stores any: d is a multiple of eight.  16384 x 2048 bf16 in 16 us
// (256 columns to a warp: 30), a tiled table's 8192 x 1024 in 6 us (bit by bit with a division each: 24).
template <typename ROWS, typename YT>
__global__ void __launch_bounds__(kThreads)
lookup_kernel(const LookupArgs a, const ROWS rows, int32_t segs)
{
    pdl_wait();
    const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int64_t t = segs == 1 ? w : w / segs;
    if (t >= a.T) return;
    const int32_t c0 = (int32_t)(w - t * segs) * 1024 + (threadIdx.x & 31) * 8;
    const int64_t id = a.ids[t];
    const bool in = inside(id, a.V, a.padding);
    YT *y = static_cast<YT *>(a.y) + t * a.d;
    const typename ROWS::Row row = rows.row(in ? id : 0);
    typename ROWS::Piece p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (in && c0 + i * 256 < a.d) rows.load(row, c0 + i * 256, p[i]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (c0 + i * 256 >= a.d) break;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (in) rows.values(row, c0 + i * 256, p[i], v);
        store_row(y + c0 + i * 256, v);
    }
}

// Other rows: y as one array, an aligned piece of eight to a thread.  (Several to a thread: 8192 x 2047 bf16 5 to 15 us slower.)  The values of
// a piece that lies in two rows are asked for together, one by one where rows are shorter than a piece.
template <typename ROWS, typename YT>
__global__ void __launch_bounds__(kThreads)
lookup_odd_kernel(const LookupArgs a, const ROWS rows)
{
    pdl_wait();
    const int64_t o = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 8, total = a.T * a.d;
    if (o >= total) return;
    YT *y = static_cast<YT *>(a.y);
    int64_t t = total <= 0x7fffffff ? (int64_t)((uint32_t)o / (uint32_t)a.d) : o / a.d;
    int32_t c = (int32_t)(o - t * a.d);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    int64_t id = a.ids[t];
    if (c + 8 <= a.d) {
        if (inside(id, a.V, a.padding)) {
            const typename ROWS::Row row = rows.row(id);
            typename ROWS::Piece p;
            rows.load(row, c, p);
            rows.values(row, c, p, v);
        }
        store_row(y + o, v);
    } else if (a.d >= 8) {
        const int32_t here = a.d - c;                                 // of the first row; the rest is the next one's, if there is one
        const int64_t id2 = t + 1 < a.T ? a.ids[t + 1] : -1;
        const bool in = inside(id, a.V, a.padding), in2 = inside(id2, a.V, a.padding);
        const typename ROWS::Row row = rows.row(in ? id : 0), row2 = rows.row(in2 ? id2 : 0);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e < here) { if (in) v[e] = rows.one(row, c + e); }
            else if (in2) v[e] = rows.one(row2, e - here);
        }
        if (o + 8 <= total) store_row(y + o, v);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) if (o + e < total) store_from_float(y, o + e, v[e]);
    } else {
        for (int e = 0; e < 8 && o + e < total; ++e) {
            store_from_float(y, o + e, inside(id, a.V, a.padding) ? rows.one(rows.row(id), c) : 0.0f);
            if (++c == a.d) {
                c = 0;
                ++t;
                id = t < a.T ? a.ids[t] : -1;
            }
        }
    }
}

// ---- tokens sorted by id ---------------------------------------------------------------------------------------------------
// Least significant digit first; a thread block takes a stretch of the list (a part).  A pass needs, for each part and digit, how many
// tokens of smaller digits there are anywhere, and of this digit in the parts before: every block adds that up itself from the
// parts' counts, which the pass before left (the first pass's: count_kernel).  What lies between the passes is one launch each.
constexpr int kMaxBins = 1024;
constexpr int kSortWarps = kThreads / 32;

struct Sort {
    const int64_t *ids;
    int64_t T;
    int32_t V;
    int64_t padding;
    int32_t part;                           // tokens to a part: a multiple of kThreads
    int32_t parts;
    int32_t bits;                           // of a digit
    int32_t passes;
    uint2 *list[2];                         // (id, token)
    uint32_t *count[2];                     // [parts][bins]: of the pass that comes, of the one after it
};
// Zeros over a stretch of dw beside the sort, which keeps few of the SMs busy.
struct Fill {
    char *to;
    int64_t bytes;                          // a multiple of 2
};

__device__ __forceinline__ uint32_t key_of(const Sort &s, int64_t t)
{
    const int64_t id = s.ids[t];
    return inside(id, s.V, s.padding) ? (uint32_t)id : (uint32_t)s.V;           // what is outside goes to the end
}
template <int THREADS> __device__ __forceinline__ void fill(const Fill &f, unsigned block, unsigned blocks)
{
    const int64_t whole = f.bytes / 16;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int64_t i = (int64_t)block * THREADS + threadIdx.x; i < whole; i += (int64_t)blocks * THREADS) reinterpret_cast<uint4 *>(f.to)[i] = zero;
    if (block == 0)
        for (int64_t i = whole * 8 + threadIdx.x; i < f.bytes / 2; i += THREADS) reinterpret_cast<uint16_t *>(f.to)[i] = 0;
}

// The lanes that are `here` with the same digit of `bits` bits, one vote for each bit (4096 tokens: 2.1 us less a pass than
// __match_any_sync).
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, int bits, bool here)
{
    uint32_t same = __ballot_sync(0xffffffffu, here);
    for (int b = 0; b < bits; ++b) {
        const bool one = digit >> b & 1u;
        const uint32_t v = __ballot_sync(0xffffffffu, one);
        same &= one ? v : ~v;
    }
    return same;
}

__global__ void __launch_bounds__(kThreads)
count_kernel(const Sort s, const Fill f)
{
    __shared__ uint32_t bin[kMaxBins];
    pdl_wait();
    if (blockIdx.x >= (unsigned)s.parts) { fill<kThreads>(f, blockIdx.x - s.parts, gridDim.x - s.parts); return; }
    const int bins = 1 << s.bits;
    for (int b = threadIdx.x; b < bins; b += kThreads) bin[b] = 0;
    __syncthreads();
    const int64_t t0 = (int64_t)blockIdx.x * s.part, t1 = t0 + s.part < s.T ? t0 + s.part : s.T;
    for (int64_t t = t0 + threadIdx.x; t < t1; t += kThreads) atomicAdd(&bin[key_of(s, t) & (uint32_t)(bins - 1)], 1u);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += kThreads) {
        s.count[0][(int64_t)blockIdx.x * bins + b] = bin[b];
        if (s.passes > 1) s.count[1][(int64_t)blockIdx.x * bins + b] = 0;
    }
}

// Pass `pass` from list[pass & 1] (the first: from the ids) to list[~pass & 1].
__global__ void __launch_bounds__(kThreads)
place_kernel(const Sort s, int32_t pass, const Fill f)
{
    __shared__ uint32_t base[kMaxBins];                               // where the part's first token of a digit goes
    __shared__ uint32_t seen[kSortWarps][kMaxBins];                   // tokens of a digit, per warp: counts, then places
    __shared__ uint32_t warp_total[kSortWarps];
    pdl_wait();
    if (blockIdx.x >= (unsigned)s.parts) { fill<kThreads>(f, blockIdx.x - s.parts, gridDim.x - s.parts); return; }
    const int bins = 1 << s.bits, shift = pass * s.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t *count = s.count[pass & 1];
    uint32_t *next = s.count[(pass + 1) & 1];
    const uint2 *from = s.list[pass & 1];
    uint2 *to = s.list[(pass + 1) & 1];

    // digits in order: thread i takes bins i * per ... of them
    const int per = (bins + kThreads - 1) / kThreads;
    uint32_t total[kMaxBins / kThreads], before[kMaxBins / kThreads], sum = 0;
#pragma unroll
    for (int j = 0; j < kMaxBins / kThreads; ++j) {
        total[j] = before[j] = 0;
        const int b = threadIdx.x * per + j;
        if (j < per && b < bins)
#pragma unroll 8
            for (int32_t p = 0; p < s.parts; ++p) {
                const uint32_t c = count[(int64_t)p * bins + b];
                total[j] += c;
                if (p < (int32_t)blockIdx.x) before[j] += c;
            }
        sum += total[j];
    }
    uint32_t run = sum;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, run, off);
        if (lane >= off) run += o;
    }
    if (lane == 31) warp_total[warp] = run;
    for (int b = threadIdx.x; b < kSortWarps * kMaxBins; b += kThreads) (&seen[0][0])[b] = 0;
    __syncthreads();
    run -= sum;
    for (int w = 0; w < warp; ++w) run += warp_total[w];
#pragma unroll
    for (int j = 0; j < kMaxBins / kThreads; ++j) {
        const int b = threadIdx.x * per + j;
        if (j < per && b < bins) base[b] = run + before[j];
        run += total[j];
    }

    // the part's tokens: a warp takes a stretch of them, and keeps their order
    const int64_t t0 = (int64_t)blockIdx.x * s.part, t1 = t0 + s.part < s.T ? t0 + s.part : s.T;
    const int64_t w0 = t0 + (int64_t)warp * (s.part / kSortWarps);
    int64_t w1 = w0 + s.part / kSortWarps;
    if (w1 > t1) w1 = t1;
    // four rounds at a time, whose tokens are asked for together
    auto items = [&](int64_t tb, uint2 (&item)[4]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t t = tb + r * 32 + lane;
            item[r] = make_uint2(0, 0);
            if (t < w1) item[r] = pass == 0 ? make_uint2(key_of(s, t), (uint32_t)t) : from[t];
        }
    };
    for (int64_t tb = w0; tb < w1; tb += 128) {
        uint2 item[4];
        items(tb, item);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (tb + r * 32 + lane < w1) atomicAdd(&seen[warp][(item[r].x >> shift) & (uint32_t)(bins - 1)], 1u);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += kThreads) {
        uint32_t at = base[b];
        for (int w = 0; w < kSortWarps; ++w) { const uint32_t c = seen[w][b]; seen[w][b] = at; at += c; }
    }
    __syncthreads();
    for (int64_t tb = w0; tb < w1; tb += 128) {
        uint2 four[4];
        items(tb, four);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (tb + r * 32 >= w1) break;
            const bool here = tb + r * 32 + lane < w1;
            const uint2 item = four[r];
            const uint32_t digit = (item.x >> shift) & (uint32_t)(bins - 1), same = same_digit(digit, s.bits, here);
            const uint32_t rank = __popc(same & ((1u << lane) - 1u));
            uint32_t at = 0;
            if (here) at = seen[warp][digit] + rank;
            __syncwarp();
            if (here && rank == 0) seen[warp][digit] += __popc(same);
            __syncwarp();
            if (here) {
                to[at] = item;
                if (pass + 1 < s.passes)
                    atomicAdd(&next[(int64_t)(at / (uint32_t)s.part) * bins + ((item.x >> (shift + s.bits)) & (uint32_t)(bins - 1))], 1u);
            }
        }
    }
}

// next's next: the counts of pass + 2 go where this pass's are, so they are cleared between the two (three passes and more only)
__global__ void __launch_bounds__(kThreads)
clear_kernel(uint32_t *__restrict__ count, int64_t n)
{
    pdl_wait();
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) count[i] = 0;
}

// Few tokens are sorted in one launch, by counting: a token goes behind all with a smaller id and those before it with its own.  A thread
// block takes 32 tokens, one to a lane, and its warps a share of the list each; T^2 comparisons, at two instructions for 32 of them, spread over
// the SMs (4096 tokens: 5.9 us within a step; by itself 7.8, where one thread block sorting by digits took 13.8 and the launches above 19).
constexpr int kRankTokens = 8192;
__global__ void __launch_bounds__(kThreads)
rank_kernel(const Sort s, const Fill f, unsigned rankers)
{
    extern __shared__ __align__(16) char smem[];
    uint32_t *key = reinterpret_cast<uint32_t *>(smem);               // T of them, then ones beyond every key up to a multiple of 4
    __shared__ uint32_t part[kSortWarps][32];
    pdl_wait();
    if (blockIdx.x >= rankers) { fill<kThreads>(f, blockIdx.x - rankers, gridDim.x - rankers); return; }
    const int T = (int)s.T, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int padded = (T + 31) & ~31;
#pragma unroll 16
    for (int t = threadIdx.x; t < padded; t += kThreads) key[t] = t < T ? key_of(s, t) : 0xffffffffu;
    __syncthreads();
    const int t0 = blockIdx.x * 32;
    const uint32_t mine = key[t0 + lane];
    uint32_t count = 0;
    // the list in groups of 32: those before the block's own count where not larger, those behind it where smaller
    const int groups = padded / 32, own = blockIdx.x;
    for (int g = warp; g < groups; g += kSortWarps) {
        const uint4 *k4 = reinterpret_cast<const uint4 *>(key + g * 32);
        const uint32_t limit = mine + (g < own ? 1u : 0u);            // not larger: smaller than the next number
        if (g != own) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint4 k = k4[i];
                count += (k.x < limit) + (k.y < limit) + (k.z < limit) + (k.w < limit);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t k = key[t0 + i];
                count += k < mine || (k == mine && i < lane);
            }
        }
    }
    part[warp][lane] = count;
    __syncthreads();
    if (warp == 0 && t0 + lane < T) {
#pragma unroll
        for (int w = 1; w < kSortWarps; ++w) count += part[w][lane];
        s.list[0][count] = make_uint2(mine, (uint32_t)(t0 + lane));
    }
}

// ---- sums -------------------------------------------------------------------------------------------------------------------
// Columns of a row of dw are taken in the aligned pieces that cover it: piece c / 8 begins at column c - shift, shift = (id d) mod 8 (0 where
// d is a multiple of eight: EVEN).  The same columns of dy's rows begin anywhere.
template <bool EVEN> __device__ __forceinline__ int32_t shift_of(uint32_t id, int32_t d) { return EVEN ? 0 : (int32_t)((id * (uint32_t)d) & 7u); }
template <bool EVEN> __device__ __forceinline__ bool all_in(int32_t c, int32_t d) { return EVEN ? c < d : c >= 0 && c + 8 <= d; }
template <bool EVEN> __device__ __forceinline__ bool some_in(int32_t c, int32_t d) { return EVEN ? c < d : c > -8 && c < d; }

// A row's columns of a piece at its ends, zeros beside them; all asked for together.
template <typename T> __device__ __forceinline__ void load_part(const T *row, int32_t c, int32_t d, Raw8<T> &r)
{
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = c + e >= 0 && c + e < d ? __float_as_uint(value_of(row[c + e])) : 0u;
    if (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.w[e % (int)(sizeof(r.w) / 4)] = h[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) r.w[e] = h[2 * e] >> 16 | (h[2 * e + 1] & 0xffff0000u);
    }
}
// A lane's eight columns of a row of dw, from column c on: what was there (`old`, loaded ahead) and the sum, written.
template <bool EVEN, bool ADD, typename WT>
__device__ __forceinline__ void write_sum(WT *row, int32_t c, int32_t d, const float (&acc)[8], float scale, const Raw8<WT> &old)
{
    if (!some_in<EVEN>(c, d)) return;
    float o[8];
    if (ADD) unpack8(old, o);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = ADD ? fmaf(scale, acc[e], o[e]) : scale * acc[e];
    if (all_in<EVEN>(c, d)) store_row(row + c, o);
    else
#pragma unroll
        for (int e = 0; e < 8; ++e) if (c + e >= 0 && c + e < d) store_from_float(row, c + e, o[e]);
}
// Sums of pieces lie in rows of `pitch` floats (a multiple of eight).
__device__ __forceinline__ void put_partial(float *row, int32_t c, const float (&acc)[8]) { store_row(row + c, acc); }

// A warp takes one piece of the sorted list and NP * 256 columns.  An id's tokens that begin and end in the piece are done with; what
// comes from the piece before, or goes on in the next one, is written to `partial` ([piece][2][pitch]: first, last).  16384 x 2048 bf16 over
// 50021 ids: 23 us within a step, 17 by itself (1024 columns to a warp; with 256 34); 4096 x 1024 added to fp32: 6.4 and 8 (11 with rows of
// dw read where a sum ends).
template <typename GT, typename WT, int NP, bool EVEN, bool ADD>
__global__ void __launch_bounds__(kThreads)
sum_kernel(const uint2 *__restrict__ list, int64_t T, int32_t V, int32_t d, int32_t piece, int64_t pieces, int32_t segs, float scale,
           const GT *__restrict__ dy, WT *dw, float *__restrict__ partial, int32_t pitch)
{
    // Rows of dy loaded before the first is added, with the rows of dw that sums beginning there will be added to: more of them hide more of
    // each load and leave fewer warps to an SM (us, with 2 / 4 / 8: 16384 x 2048 bf16 added 65 / 64 / 73).  Odd bf16 rows have two pieces on
    // their way for each (us, with 2 / 4: added 16384 x 2047 98 / 114, 32768 x 1023 108 / 133, 9000 x 1500 46 / 54, 32768 x 63 53 / 54; as a
    // whole table 104 / 112, 98 / 96, 84 / 84, 50 / 49).
    constexpr int kAhead = NP == 1 ? (EVEN || sizeof(GT) == 4 ? 4 : 2) : sizeof(GT) == 2 ? 8 / NP * 2 : 8 / NP;
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int64_t k = segs == 1 ? w : w / segs;
    if (k >= pieces) return;
    const int32_t c0 = (int32_t)(w - k * segs) * (256 * NP) + lane * 8;
    const int64_t a = k * piece;
    const int n = (int)(T - a < piece ? T - a : piece);
    const GT *end = dy + T * d;
    uint2 item = make_uint2(0xffffffffu, 0);
    if (lane < n) item = list[a + lane];
    const uint32_t left = a > 0 ? list[a - 1].x : 0xffffffffu, right = a + n < T ? list[a + n].x : 0xffffffffu;
    float acc[NP][8];
    Raw8<WT> old[NP];
    uint32_t cur = 0xffffffffu;
    bool from_left = false;
    auto put = [&](bool to_right) {
        if (cur >= (uint32_t)V) return;
        if (from_left || to_right) {
            float *row = partial + (k * 2 + (from_left ? 0 : 1)) * pitch;
#pragma unroll
            for (int j = 0; j < NP; ++j) if (c0 + j * 256 < pitch) put_partial(row, c0 + j * 256, acc[j]);
        } else {
            WT *row = dw + (int64_t)cur * d;
            const int32_t shift = shift_of<EVEN>(cur, d);
#pragma unroll
            for (int j = 0; j < NP; ++j) write_sum<EVEN, ADD>(row, c0 + j * 256 - shift, d, acc[j], scale, old[j]);
        }
    };
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += kAhead) {
        if (i0 > 0 && (i0 & 31) == 0) {
            item = make_uint2(0xffffffffu, 0);
            if (i0 + lane < n) item = list[a + i0 + lane];
        }
        OddPiece<GT, EVEN> r[kAhead][NP];
        Raw8<WT> there[ADD ? kAhead : 1][NP];
        uint32_t before = cur;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t key = __shfl_sync(0xffffffffu, item.x, (i0 + i) & 31), tok = __shfl_sync(0xffffffffu, item.y, (i0 + i) & 31);
            const bool starts = key != before;
            before = key;
            if (key >= (uint32_t)V) continue;                         // beyond the piece: a key of 2^32 - 1
            const int32_t shift = shift_of<EVEN>(key, d);
            if (ADD && starts) {
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    const int32_t c = c0 + j * 256 - shift;
                    if (all_in<EVEN>(c, d)) load_row(dw + (int64_t)key * d + c, there[ADD ? i : 0][j]);
                    else if (some_in<EVEN>(c, d)) load_part(dw + (int64_t)key * d, c, d, there[ADD ? i : 0][j]);
                }
            }
            const GT *row = dy + (int64_t)tok * d;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int32_t c = c0 + j * 256 - shift;
                if (all_in<EVEN>(c, d)) {
                    r[i][j].ask(row + c, end);
                } else if (!EVEN && some_in<EVEN>(c, d)) {
                    load_part(row, c, d, r[i][j].r);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t key = __shfl_sync(0xffffffffu, item.x, (i0 + i) & 31), tok = EVEN ? 0 : __shfl_sync(0xffffffffu, item.y, (i0 + i) & 31);
            if (i0 + i >= n) break;
            const bool starts = key != cur;
            if (starts) {
                put(false);
                from_left = i0 + i == 0 && key == left;
                cur = key;
                if (ADD) {
#pragma unroll
                    for (int j = 0; j < NP; ++j) old[j] = there[ADD ? i : 0][j];
                }
            }
            if (key >= (uint32_t)V) continue;
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                const int32_t c = c0 + j * 256 - shift_of<EVEN>(key, d);
                if (!some_in<EVEN>(c, d)) continue;
                float v[8];
                unpack8(!EVEN && all_in<EVEN>(c, d) ? r[i][j].take(dy + (int64_t)tok * d + c, end) : r[i][j].r, v);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[j][e] = starts ? v[e] : acc[j][e] + v[e];
            }
        }
    }
    put(cur == right);
}

// The ids whose tokens lie in several pieces.  A warp looks at one piece: does its last id begin in it and go on?  Short runs it
// adds up by itself, long ones are shared by the block's warps.  A chain of dependent reads (list, pieces, sums): 4 us at 4096 x 1024, 6 to 11
// above 8192 tokens.
constexpr int kAlone = 16;
template <typename WT, bool EVEN, bool ADD>
__global__ void __launch_bounds__(kThreads)
join_kernel(const uint2 *__restrict__ list, int64_t T, int32_t V, int32_t d, int32_t piece, int64_t pieces, float scale, WT *dw,
            const float *__restrict__ partial, int32_t pitch)
{
    constexpr int kWarps = kThreads / 32;
    __shared__ int64_t more[kWarps];                                  // pieces after the warp's own that the run covers
    __shared__ uint32_t key_at[kWarps];
    __shared__ float red[kWarps][256];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t k = (int64_t)blockIdx.x * kWarps + warp;
    const int32_t c = blockIdx.y * 256 + lane * 8;
    int64_t n = 0;
    uint32_t key = 0xffffffffu;
    if (k + 1 < pieces) {
        const int64_t a = k * piece, b = a + piece;                   // b < T: another piece follows
        const uint32_t first = list[a].x, next = list[b].x, before = a > 0 ? list[a - 1].x : 0xffffffffu;
        const int64_t o1 = k + 2 + lane;                              // the pieces after the next one, of which it is the first id
        const uint32_t ahead = o1 < pieces ? list[o1 * piece].x : 0xffffffffu;
        key = list[b - 1].x;
        if (key < (uint32_t)V && next == key && (first != key || before != key)) {
            uint32_t off = __ballot_sync(0xffffffffu, ahead != key);
            n = 1;
            while (off == 0) {
                n += 32;
                const int64_t o = k + 1 + n + lane;
                off = __ballot_sync(0xffffffffu, !(o < pieces && list[o * piece].x == key));
            }
            n += __ffs(off) - 1;
        }
    }
    auto add_up = [&](int64_t from, int64_t lo, int64_t hi, float (&acc)[8]) {          // partials lo .. hi of the run of piece `from`
        if (c >= pitch) return;
        int64_t i = lo;
        for (; i + 8 <= hi; i += 8) {
            Raw8<float> r[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) load_row(partial + ((from + i + j) * 2 + (i + j == 0 ? 1 : 0)) * pitch + c, r[j]);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] += __uint_as_float(r[j].w[e]);
        }
        for (; i < hi; ++i) {
            Raw8<float> r;
            load_row(partial + ((from + i) * 2 + (i == 0 ? 1 : 0)) * pitch + c, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += __uint_as_float(r.w[e]);
        }
    };
    auto row_there = [&](uint32_t id, Raw8<WT> &old) {
        const int32_t at = c - shift_of<EVEN>(id, d);
        if (ADD && all_in<EVEN>(at, d)) load_row(dw + (int64_t)id * d + at, old);
        else if (ADD && some_in<EVEN>(at, d)) load_part(dw + (int64_t)id * d, at, d, old);
    };
    if (n > 0 && n <= kAlone) {
        float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        Raw8<WT> old;
        row_there(key, old);
        add_up(k, 0, n + 1, acc);
        write_sum<EVEN, ADD>(dw + (int64_t)key * d, c - shift_of<EVEN>(key, d), d, acc, scale, old);
    }
    if (lane == 0) { more[warp] = n > kAlone ? n : 0; key_at[warp] = key; }
    __syncthreads();
    for (int j = 0; j < kWarps; ++j) {
        const int64_t len = more[j] + 1;                              // the same for the whole block
        if (len == 1) continue;
        float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        Raw8<WT> old;
        if (warp == 0) row_there(key_at[j], old);
        add_up((int64_t)blockIdx.x * kWarps + j, len * warp / kWarps, len * (warp + 1) / kWarps, acc);
#pragma unroll
        for (int e = 0; e < 8; ++e) red[warp][e * 32 + lane] = acc[e];
        __syncthreads();
        if (warp == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                for (int i = 1; i < kWarps; ++i) acc[e] += red[i][e * 32 + lane];
            write_sum<EVEN, ADD>(dw + (int64_t)key_at[j] * d, c - shift_of<EVEN>(key_at[j], d), d, acc, scale, old);
        }
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kThreads)
zero_kernel(const Fill f)
{
    pdl_wait();
    fill<kThreads>(f, blockIdx.x, gridDim.x);
}

// ---- host side ----------------------------------------------------------------------------------------------------------------
size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

struct Plan {
    int32_t part, parts, bits, passes, piece, pitch;
    bool one;                               // sorted in one launch
    int64_t pieces;
    size_t o_list[2], o_count[2], o_partial, total;
};
Plan make_plan(int64_t T, int32_t d, int32_t V)
{
    Plan p = {};
    int32_t need = 1;
    while (((int64_t)V >> need) != 0) ++need;                         // bits of V, the key of what is outside
    p.one = T <= kRankTokens;
    p.passes = (need + 9) / 10;
    p.bits = (need + p.passes - 1) / p.passes;
    // parts of 1024 tokens: four rounds of a block's warps; more when the blocks' sums over all parts' counts would grow
    int64_t part = 1024;
    const int64_t most = 128;
    if ((T + part - 1) / part > most) part = (int64_t)round_up((size_t)((T + most - 1) / most), kThreads);
    p.part = (int32_t)part;
    p.parts = (int32_t)((T + part - 1) / part);
    p.piece = T <= 4096 ? 8 : T <= 32768 ? 16 : T <= 131072 ? 32 : 64;
    p.pieces = (T + p.piece - 1) / p.piece;
    p.pitch = (d % 8 ? d + 7 : d) / 8 * 8 + (d % 8 ? 8 : 0);         // whole pieces that a row can touch
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += round_up(bytes, 256); return at; };
    p.o_list[0] = take((size_t)T * sizeof(uint2));
    if (!p.one) {
        p.o_list[1] = take((size_t)T * sizeof(uint2));
        for (int i = 0; i < 2; ++i) p.o_count[i] = take((size_t)p.parts << (p.bits + 2));
    }
    p.o_partial = take(p.pieces > 1 ? (size_t)p.pieces * 2 * p.pitch * 4 : 0);
    p.total = o;
    return p;
}

template <typename YT, typename ROWS> cudaError_t lookup_even(const LookupArgs &a, const ROWS &rows, cudaStream_t s)
{
    const int32_t segs = (a.d + 1023) / 1024;
    const int64_t blocks = (a.T * segs + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_pdl(lookup_kernel<ROWS, YT>, dim3((unsigned)blocks), dim3(kThreads), 0, s, a, rows, segs);
}
template <typename YT, typename ROWS> cudaError_t lookup_odd(const LookupArgs &a, const ROWS &rows, cudaStream_t s)
{
    const int64_t blocks = (a.T * a.d + kThreads * 8 - 1) / (kThreads * 8);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_pdl(lookup_odd_kernel<ROWS, YT>, dim3((unsigned)blocks), dim3(kThreads), 0, s, a, rows);
}
template <typename WT, typename YT> cudaError_t lookup_typed(const LookupArgs &a, cudaStream_t s)
{
    if (a.table) {
        const WT *table = static_cast<const WT *>(a.table);
        const WT *end = table + (int64_t)a.V * a.d;
        return a.d % 8 == 0 ? lookup_even<YT>(a, DenseRows<WT, true>{table, end, a.d, a.scale}, s)
                            : lookup_odd<YT>(a, DenseRows<WT, false>{table, end, a.d, a.scale}, s);
    }
    const int32_t rows = a.q % a.d == 0 ? (int32_t)(a.q / a.d) : 0;
    const TiledRows tiled = {a.tile, a.alpha, a.q, (a.q + 31) / 32, a.d, rows, a.per_tile, a.scale};
    return a.d % 8 == 0 ? lookup_even<YT>(a, tiled, s) : lookup_odd<YT>(a, tiled, s);
}

template <typename GT, typename WT, int NP, bool EVEN, bool ADD>
cudaError_t sum_pieces(const GradArgs &a, const Plan &p, const uint2 *list, float *partial, cudaStream_t s)
{
    const int32_t segs = (p.pitch + 256 * NP - 1) / (256 * NP);
    const int64_t blocks = (p.pieces * segs + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
    return launch_pdl(sum_kernel<GT, WT, NP, EVEN, ADD>, dim3((unsigned)blocks), dim3(kThreads), 0, s, list, a.T, a.V, a.d, p.piece, p.pieces, segs, a.scale,
                      static_cast<const GT *>(a.dy), static_cast<WT *>(a.dw), partial, p.pitch);
}
template <typename GT, typename WT, bool EVEN, bool ADD>
cudaError_t sums(const GradArgs &a, const Plan &p, const uint2 *list, float *partial, cudaStream_t s)
{
    // The more columns to a warp the less a row costs, while there are warps for every SM and registers for the rows on their way.  Odd rows,
    // and sums with dw's rows beside them, are fastest with one piece to a lane (us, one / two pieces: dense 16384 x 2047 bf16 104 / 128,
    // added 98 / 181, 16384 x 2048 added 64 / 67).
    const int64_t warps = (int64_t)sm_count() * 12;
    cudaError_t e = cudaErrorNotReady;
    if constexpr (EVEN && !ADD) {
        if (a.d > 512 && p.pieces * ((a.d + 1023) / 1024) >= warps) e = sum_pieces<GT, WT, 4, EVEN, ADD>(a, p, list, partial, s);
        else if (a.d > 256 && p.pieces * ((a.d + 511) / 512) >= warps) e = sum_pieces<GT, WT, 2, EVEN, ADD>(a, p, list, partial, s);
    }
    if (e == cudaErrorNotReady) e = sum_pieces<GT, WT, 1, EVEN, ADD>(a, p, list, partial, s);
    if (e != cudaSuccess || p.pieces == 1) return e;
    const int32_t segs = (p.pitch + 255) / 256;
    return launch_pdl(join_kernel<WT, EVEN, ADD>, dim3((unsigned)((p.pieces + kThreads / 32 - 1) / (kThreads / 32)), (unsigned)segs), dim3(kThreads), 0, s,
                      list, a.T, a.V, a.d, p.piece, p.pieces, a.scale, static_cast<WT *>(a.dw), static_cast<const float *>(partial), p.pitch);
}
template <typename GT, typename WT> cudaError_t sums_typed(const GradArgs &a, const Plan &p, const uint2 *list, float *partial, cudaStream_t s)
{
    if (a.d % 8 == 0) return a.add ? sums<GT, WT, true, true>(a, p, list, partial, s) : sums<GT, WT, true, false>(a, p, list, partial, s);
    return a.add ? sums<GT, WT, false, true>(a, p, list, partial, s) : sums<GT, WT, false, false>(a, p, list, partial, s);
}

}  // namespace

int lookup(const LookupArgs &a, cudaStream_t s)
{
    cudaError_t e;
    if (!a.table || a.table_dtype == TBN_F32) e = a.y_dtype == TBN_F32 ? lookup_typed<float, float>(a, s) : lookup_typed<float, __nv_bfloat16>(a, s);
    else e = a.y_dtype == TBN_F32 ? lookup_typed<__nv_bfloat16, float>(a, s) : lookup_typed<__nv_bfloat16, __nv_bfloat16>(a, s);
    return e == cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
}

size_t gradient_workspace_bytes(int64_t T, int32_t d, int32_t V) { return make_plan(T, d, V).total; }

int gradient(const GradArgs &a, void *workspace, cudaStream_t s)
{
    const int64_t dw_bytes = (int64_t)a.V * a.d * (a.dw_dtype == TBN_BF16 ? 2 : 4);
    const unsigned fillers = (unsigned)sm_count() * 4;
    if (a.T == 0) {
        if (a.add) return TBN_OK;
        return launch_pdl(zero_kernel, dim3(fillers), dim3(kThreads), 0, s, Fill{static_cast<char *>(a.dw), dw_bytes}) == cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
    }
    const Plan p = make_plan(a.T, a.d, a.V);
    char *ws = static_cast<char *>(workspace);
    Sort so = {};
    so.ids = a.ids; so.T = a.T; so.V = a.V; so.padding = a.padding; so.part = p.part; so.parts = p.parts; so.bits = p.bits; so.passes = p.passes;
    for (int i = 0; i < 2; ++i) {
        so.list[i] = reinterpret_cast<uint2 *>(ws + p.o_list[i]);
        so.count[i] = reinterpret_cast<uint32_t *>(ws + p.o_count[i]);
    }
    const uint2 *list = so.list[0];
    if (p.one) {
        const Fill f = {static_cast<char *>(a.dw), a.add ? 0 : dw_bytes};
        const unsigned rankers = (unsigned)((a.T + 31) / 32);
        const int64_t blocks = (dw_bytes + 16383) / 16384;
        const unsigned grid = rankers + (a.add ? 0u : (unsigned)(blocks < fillers ? blocks : fillers));
        if (launch_spread(rank_kernel, dim3(grid), dim3(kThreads), (size_t)rankers * 128, s, so, f, rankers) != cudaSuccess) return TBN_ERR_CUDA;
    } else {
        // the zeros, in as many equal stretches as the sort has launches
        const int launches = p.passes + 1;
        const int64_t share = (dw_bytes / launches + 15) / 16 * 16;
        auto stretch = [&](int i) {
            const int64_t lo = share * i < dw_bytes ? share * i : dw_bytes, hi = i == launches - 1 ? dw_bytes : lo + share < dw_bytes ? lo + share : dw_bytes;
            return a.add ? Fill{static_cast<char *>(a.dw), 0} : Fill{static_cast<char *>(a.dw) + lo, hi - lo};
        };
        const dim3 grid((unsigned)p.parts + (a.add ? 0u : fillers));
        if (launch_spread(count_kernel, grid, dim3(kThreads), 0, s, so, stretch(0)) != cudaSuccess) return TBN_ERR_CUDA;
        for (int i = 0; i < p.passes; ++i) {
            if (launch_pdl(place_kernel, grid, dim3(kThreads), 0, s, so, i, stretch(i + 1)) != cudaSuccess) return TBN_ERR_CUDA;
            if (i + 2 < p.passes &&
                launch_pdl(clear_kernel, dim3(64), dim3(kThreads), 0, s, so.count[i & 1], (int64_t)p.parts << p.bits) != cudaSuccess)
                return TBN_ERR_CUDA;
        }
        list = so.list[p.passes & 1];
    }
    float *partial = reinterpret_cast<float *>(ws + p.o_partial);
    cudaError_t e;
    if (a.dy_dtype == TBN_F32) e = a.dw_dtype == TBN_F32 ? sums_typed<float, float>(a, p, list, partial, s) : sums_typed<float, __nv_bfloat16>(a, p, list, partial, s);
    else e = a.dw_dtype == TBN_F32 ? sums_typed<__nv_bfloat16, float>(a, p, list, partial, s) : sums_typed<__nv_bfloat16, __nv_bfloat16>(a, p, list, partial, s);
    return e == cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
}

}  // namespace embed
}  // namespace tbn
