// Embedding lookup with scaling, from a table or from a tiled table's bits, and the table's gradient.
//
//   y_t = scale table[id_t],   dw_v = scale sum_{t: id_t = v} dy_t     (ids outside the vocabulary: y_t = 0, no gradient)
//
// Both are bound by HBM.  The gradient adds rows in the order of the tokens, whatever the GPU does first: the tokens are sorted by
// id (stable, by digits of the id), equal pieces of the sorted list are summed by a warp each, 256 columns at a time, and where an
// id's tokens go on over several pieces the pieces' sums are added in order by a kernel of their own.  No row of dy is read
// twice, no atomic decides an order.
#include "embedding.cuh"
#include "vec8.cuh"

namespace tbn {
namespace embed {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ bool inside(int64_t id, int32_t V, int64_t padding) { return id >= 0 && id < V && id != padding; }

// Columns of a lane within 256 of a row: eight in a row (VEC) or every 32nd.
template <bool VEC, typename T> __device__ __forceinline__ void load_cols(const T *row, int32_t c0, int32_t d, float (&v)[8])
{
    const int lane = threadIdx.x & 31;
    if (VEC) {
        if (c0 + lane * 8 < d) { unpack8(load8(row + c0 + lane * 8), v); return; }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c0 + lane + 32 * e < d ? value_of(row[c0 + lane + 32 * e]) : 0.0f;
    }
}
template <bool VEC, typename T> __device__ __forceinline__ void store_cols(T *row, int32_t c0, int32_t d, const float (&v)[8])
{
    const int lane = threadIdx.x & 31;
    if (VEC) {
        if (c0 + lane * 8 < d) store8(row + c0 + lane * 8, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (c0 + lane + 32 * e < d) store_from_float(row, c0 + lane + 32 * e, v[e]);
    }
}

// A warp takes 256 columns of one token.
template <typename WT, typename YT, bool VEC>
__global__ void __launch_bounds__(kThreads)
lookup_kernel(const LookupArgs a, int32_t segs)
{
    pdl_launch_dependents();
    pdl_wait();
    const int64_t warps = (int64_t)gridDim.x * (kThreads / 32), total = a.T * segs;
    for (int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); w < total; w += warps) {
        const int64_t t = w / segs;
        const int32_t c0 = (int32_t)(w - t * segs) * 256;
        const int64_t id = a.ids[t];
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (inside(id, a.V, a.padding)) {
            load_cols<VEC>(static_cast<const WT *>(a.table) + id * a.d, c0, a.d, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= a.scale;
        }
        store_cols<VEC>(static_cast<YT *>(a.y) + t * a.d, c0, a.d, v);
    }
}

template <typename YT, bool VEC>
__global__ void __launch_bounds__(kThreads)
lookup_tiled_kernel(const LookupArgs a, int32_t segs)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (kThreads / 32), total = a.T * segs;
    for (int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); w < total; w += warps) {
        const int64_t t = w / segs;
        const int32_t c0 = (int32_t)(w - t * segs) * 256;
        const int64_t id = a.ids[t];
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (inside(id, a.V, a.padding)) {
            const int64_t f0 = id * a.d + c0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int32_t c = VEC ? lane * 8 + e : lane + 32 * e;
                if (c0 + c < a.d) {
                    const int64_t f = f0 + c, j = f / a.q, i = f - j * a.q;
                    const float al = __ldg(a.alpha + (a.per_tile ? j : 0)) * a.scale;
                    v[e] = tile_bit(a.tile, i) ? al : -al;
                }
            }
        }
        store_cols<VEC>(static_cast<YT *>(a.y) + t * a.d, c0, a.d, v);
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
__device__ __forceinline__ void fill(const Fill &f, unsigned block, unsigned blocks)
{
    const int64_t whole = f.bytes / 16;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int64_t i = (int64_t)block * kThreads + threadIdx.x; i < whole; i += (int64_t)blocks * kThreads) reinterpret_cast<uint4 *>(f.to)[i] = zero;
    if (block == 0)
        for (int64_t i = whole * 8 + threadIdx.x; i < f.bytes / 2; i += kThreads) reinterpret_cast<uint16_t *>(f.to)[i] = 0;
}

__global__ void __launch_bounds__(kThreads)
count_kernel(const Sort s, const Fill f)
{
    __shared__ uint32_t bin[kMaxBins];
    pdl_launch_dependents();
    pdl_wait();
    if (blockIdx.x >= (unsigned)s.parts) { fill(f, blockIdx.x - s.parts, gridDim.x - s.parts); return; }
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
    pdl_launch_dependents();
    pdl_wait();
    if (blockIdx.x >= (unsigned)s.parts) { fill(f, blockIdx.x - s.parts, gridDim.x - s.parts); return; }
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
    for (int64_t t = w0 + lane; t < w1; t += 32) {
        const uint32_t key = pass == 0 ? key_of(s, t) : from[t].x;
        atomicAdd(&seen[warp][(key >> shift) & (uint32_t)(bins - 1)], 1u);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += kThreads) {
        uint32_t at = base[b];
        for (int w = 0; w < kSortWarps; ++w) { const uint32_t c = seen[w][b]; seen[w][b] = at; at += c; }
    }
    __syncthreads();
    for (int64_t tb = w0; tb < w1; tb += 32) {
        const int64_t t = tb + lane;
        const bool here = t < w1;
        uint2 item = make_uint2(0, 0);
        if (here) item = pass == 0 ? make_uint2(key_of(s, t), (uint32_t)t) : from[t];
        const uint32_t digit = here ? (item.x >> shift) & (uint32_t)(bins - 1) : 0xffffffffu;
        const uint32_t same = __match_any_sync(0xffffffffu, digit);
        const uint32_t rank = __popc(same & ((1u << lane) - 1u));
        uint32_t at = 0;
        if (here) at = seen[warp][digit] + rank;
        __syncwarp();
        if (here && rank == 0) seen[warp][digit] += __popc(same);
        __syncwarp();
        if (here) {
            to[at] = item;
            if (pass + 1 < s.passes) atomicAdd(&next[(int64_t)(at / (uint32_t)s.part) * bins + ((item.x >> (shift + s.bits)) & (uint32_t)(bins - 1))], 1u);
        }
    }
}

// next's next: the counts of pass + 2 go where this pass's are, so they are cleared between the two (three passes and more only)
__global__ void __launch_bounds__(kThreads)
clear_kernel(uint32_t *__restrict__ count, int64_t n)
{
    pdl_launch_dependents();
    pdl_wait();
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) count[i] = 0;
}

// ---- sums -------------------------------------------------------------------------------------------------------------------
// A warp takes one piece of the sorted list and 256 columns.  An id's tokens that begin and end in the piece are done with; what
// comes from the piece before, or goes on in the next one, is written to `partial` ([piece][2][d]: first, last).
template <typename GT, typename WT, bool VEC>
__global__ void __launch_bounds__(kThreads)
sum_kernel(const uint2 *__restrict__ list, int64_t T, int32_t V, int32_t d, int32_t piece, int64_t pieces, int32_t segs, float scale,
           const GT *__restrict__ dy, WT *__restrict__ dw, int add, float *__restrict__ partial)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int64_t c = w / segs;
    if (c >= pieces) return;
    const int32_t c0 = (int32_t)(w - c * segs) * 256;
    const int64_t a = c * piece, b = a + piece < T ? a + piece : T;
    const uint32_t left = a > 0 ? list[a - 1].x : 0xffffffffu, right = b < T ? list[b].x : 0xffffffffu;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    uint32_t cur = 0xffffffffu;
    bool from_left = false;
    auto put = [&](bool to_right) {
        if (cur >= (uint32_t)V) return;
        if (from_left || to_right) {
            store_cols<VEC>(partial + (c * 2 + (from_left ? 0 : 1)) * d, c0, d, acc);
            return;
        }
        WT *row = dw + (int64_t)cur * d;
        float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (add) load_cols<VEC>(row, c0, d, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(scale, acc[e], o[e]);
        store_cols<VEC>(row, c0, d, o);
    };
    for (int64_t p0 = a; p0 < b; p0 += 32) {
        uint2 item = make_uint2(0xffffffffu, 0);
        if (p0 + lane < b) item = list[p0 + lane];
        const int n = (int)(b - p0 < 32 ? b - p0 : 32);
        for (int i0 = 0; i0 < n; i0 += 8) {
            float v[8][8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t key = __shfl_sync(0xffffffffu, item.x, i0 + i), tok = __shfl_sync(0xffffffffu, item.y, i0 + i);
                if (i0 + i < n && key < (uint32_t)V) load_cols<VEC>(dy + (int64_t)tok * d, c0, d, v[i]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i0 + i >= n) break;
                const uint32_t key = __shfl_sync(0xffffffffu, item.x, i0 + i);
                if (key != cur) {
                    put(false);
                    from_left = p0 + i0 + i == a && key == left;
                    cur = key;
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
                }
                if (key < (uint32_t)V) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] += v[i][e];
                }
            }
        }
    }
    put(cur == right);
}

// The ids whose tokens lie in several pieces.  A warp looks at one piece: does its last id begin in it and go on?  Short runs it
// adds up by itself, long ones are shared by the block's warps.
constexpr int kAlone = 16;
template <typename WT, bool VEC>
__global__ void __launch_bounds__(kThreads)
join_kernel(const uint2 *__restrict__ list, int64_t T, int32_t V, int32_t d, int32_t piece, int64_t pieces, float scale, WT *__restrict__ dw, int add,
            const float *__restrict__ partial)
{
    constexpr int kWarps = kThreads / 32;
    __shared__ int64_t more[kWarps];                                  // pieces after the warp's own that the run covers
    __shared__ uint32_t key_at[kWarps];
    __shared__ float red[kWarps][256];
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * kWarps + warp;
    const int32_t c0 = blockIdx.y * 256;
    int64_t n = 0;
    uint32_t key = 0xffffffffu;
    if (c + 1 < pieces) {
        const int64_t a = c * piece, b = a + piece;                   // b < T: another piece follows
        key = list[b - 1].x;
        const bool begins = a == 0 || list[a].x != key || list[a - 1].x != key;
        if (key < (uint32_t)V && begins && list[b].x == key) {
            for (n = 1;; n += 32) {                                   // the pieces after the next one whose first id it is
                const int64_t o = c + 1 + n + lane;
                const bool on = o < pieces && list[o * piece].x == key;
                const uint32_t off = __ballot_sync(0xffffffffu, !on);
                if (off) { n += __ffs(off) - 1; break; }
            }
        }
    }
    auto add_up = [&](int64_t from, int64_t lo, int64_t hi, float (&acc)[8]) {          // partials lo .. hi of the run of piece `from`
        int64_t i = lo;
        for (; i + 4 <= hi; i += 4) {
            float v[4][8];
#pragma unroll
            for (int j = 0; j < 4; ++j) load_cols<VEC>(partial + ((from + i + j) * 2 + (i + j == 0 ? 1 : 0)) * d, c0, d, v[j]);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] += v[j][e];
        }
        for (; i < hi; ++i) {
            float v[8];
            load_cols<VEC>(partial + ((from + i) * 2 + (i == 0 ? 1 : 0)) * d, c0, d, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += v[e];
        }
    };
    auto finish = [&](uint32_t id, const float (&acc)[8]) {
        WT *row = dw + (int64_t)id * d;
        float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (add) load_cols<VEC>(row, c0, d, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(scale, acc[e], o[e]);
        store_cols<VEC>(row, c0, d, o);
    };
    if (n > 0 && n <= kAlone) {
        float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        add_up(c, 0, n + 1, acc);
        finish(key, acc);
    }
    if (lane == 0) { more[warp] = n > kAlone ? n : 0; key_at[warp] = key; }
    __syncthreads();
    for (int k = 0; k < kWarps; ++k) {
        const int64_t len = more[k] + 1;                              // the same for the whole block
        if (len == 1) continue;
        float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        add_up((int64_t)blockIdx.x * kWarps + k, len * warp / kWarps, len * (warp + 1) / kWarps, acc);
#pragma unroll
        for (int e = 0; e < 8; ++e) red[warp][e * 32 + lane] = acc[e];
        __syncthreads();
        if (warp == 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                for (int j = 1; j < kWarps; ++j) acc[e] += red[j][e * 32 + lane];
            finish(key_at[k], acc);
        }
        __syncthreads();
    }
}

__global__ void __launch_bounds__(kThreads)
zero_kernel(const Fill f)
{
    pdl_launch_dependents();
    pdl_wait();
    fill(f, blockIdx.x, gridDim.x);
}

// ---- host side ----------------------------------------------------------------------------------------------------------------
size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

struct Plan {
    int32_t part, parts, bits, passes, piece;
    int64_t pieces;
    size_t o_list[2], o_count[2], o_partial, total;
};
Plan make_plan(int64_t T, int32_t d, int32_t V)
{
    Plan p = {};
    int32_t need = 1;
    while (((int64_t)V >> need) != 0) ++need;                         // bits of V, the key of what is outside
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
    size_t o = 0;
    auto take = [&](size_t bytes) { const size_t at = o; o += round_up(bytes, 256); return at; };
    for (int i = 0; i < 2; ++i) p.o_list[i] = take((size_t)T * sizeof(uint2));
    for (int i = 0; i < 2; ++i) p.o_count[i] = take((size_t)p.parts << (p.bits + 2));
    p.o_partial = take((size_t)p.pieces * 2 * d * 4);
    p.total = o;
    return p;
}

template <typename WT, typename YT> cudaError_t lookup_typed(const LookupArgs &a, cudaStream_t s)
{
    const int32_t segs = (a.d + 255) / 256;
    const int64_t blocks = (a.T * segs + kThreads / 32 - 1) / (kThreads / 32), most = (int64_t)1 << 30;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    if (a.table) {
        const bool vec = aligned8<WT>(a.table, a.d) && aligned8<YT>(a.y);
        return launch_pdl(vec ? lookup_kernel<WT, YT, true> : lookup_kernel<WT, YT, false>, grid, dim3(kThreads), 0, s, a, segs);
    }
    const bool vec = aligned8<YT>(a.y, a.d);
    return launch_pdl(vec ? lookup_tiled_kernel<YT, true> : lookup_tiled_kernel<YT, false>, grid, dim3(kThreads), 0, s, a, segs);
}

template <typename GT, typename WT> cudaError_t sums_typed(const GradArgs &a, const Plan &p, const uint2 *list, float *partial, cudaStream_t s)
{
    const int32_t segs = (a.d + 255) / 256;
    const bool vec = aligned8<GT>(a.dy, a.d) && aligned8<WT>(a.dw) && aligned8<float>(partial);
    const GT *dy = static_cast<const GT *>(a.dy);
    WT *dw = static_cast<WT *>(a.dw);
    const int64_t blocks = (p.pieces * segs + kThreads / 32 - 1) / (kThreads / 32);
    cudaError_t e = launch_pdl(vec ? sum_kernel<GT, WT, true> : sum_kernel<GT, WT, false>, dim3((unsigned)blocks), dim3(kThreads), 0, s, list, a.T, a.V,
                               a.d, p.piece, p.pieces, segs, a.scale, dy, dw, a.add, partial);
    if (e != cudaSuccess || p.pieces == 1) return e;
    return launch_pdl(vec ? join_kernel<WT, true> : join_kernel<WT, false>, dim3((unsigned)((p.pieces + kThreads / 32 - 1) / (kThreads / 32)), (unsigned)segs),
                      dim3(kThreads), 0, s, list, a.T, a.V, a.d, p.piece, p.pieces, a.scale, dw, a.add, static_cast<const float *>(partial));
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
    // the zeros, in as many equal stretches as the sort has launches
    const int launches = p.passes + 1;
    const int64_t share = a.add ? 0 : (dw_bytes / launches + 15) / 16 * 16;
    auto stretch = [&](int i) {
        const int64_t lo = share * i < dw_bytes ? share * i : dw_bytes, hi = i == launches - 1 ? dw_bytes : lo + share < dw_bytes ? lo + share : dw_bytes;
        return a.add ? Fill{static_cast<char *>(a.dw), 0} : Fill{static_cast<char *>(a.dw) + lo, hi - lo};
    };
    const dim3 grid((unsigned)p.parts + (a.add ? 0u : fillers));
    if (launch_pdl(count_kernel, grid, dim3(kThreads), 0, s, so, stretch(0)) != cudaSuccess) return TBN_ERR_CUDA;
    for (int i = 0; i < p.passes; ++i) {
        if (launch_pdl(place_kernel, grid, dim3(kThreads), 0, s, so, i, stretch(i + 1)) != cudaSuccess) return TBN_ERR_CUDA;
        if (i + 2 < p.passes &&
            launch_pdl(clear_kernel, dim3(64), dim3(kThreads), 0, s, so.count[i & 1], (int64_t)p.parts << p.bits) != cudaSuccess)
            return TBN_ERR_CUDA;
    }
    const uint2 *list = so.list[p.passes & 1];
    float *partial = reinterpret_cast<float *>(ws + p.o_partial);
    cudaError_t e;
    if (a.dy_dtype == TBN_F32) e = a.dw_dtype == TBN_F32 ? sums_typed<float, float>(a, p, list, partial, s) : sums_typed<float, __nv_bfloat16>(a, p, list, partial, s);
    else e = a.dw_dtype == TBN_F32 ? sums_typed<__nv_bfloat16, float>(a, p, list, partial, s) : sums_typed<__nv_bfloat16, __nv_bfloat16>(a, p, list, partial, s);
    return e == cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
}

}  // namespace embed
}  // namespace tbn
