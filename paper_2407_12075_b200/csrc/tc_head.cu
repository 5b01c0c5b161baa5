// The contractions behind the head losses, on tcgen05 with CTA pairs.
//
//   logits   Z[t][v]  = sum_i X[t][i] W[v][i]          consumed on chip: by running maxima and sums (forward), or by the
//                                                      softmax gradient dz, which is written piece by piece (backward)
//   dX[t][i] (+)= sum_v dz[t][v] W[v][i]               dz K-major, W with its output index contiguous
//   dW[v][i]  = sum_t dz[t][v] X[t][i]                 both operands with their output index contiguous
//
// Every operand stays in the row-major form it has in memory: "K-major" and "MN-major" are the two operand forms of
// tcgen05.mma, chosen by descriptor bits, so no product needs a transposed copy.
//
// A pair of CTAs (cta_group::2) computes a 256 x 256 tile: each CTA stages 128 rows of A and 128 of B per 64-element
// step, so a byte staged feeds twice the multiplications of a 128 x 256 tile on one CTA (per 64-element step and SM:
// 32 KB instead of 48 KB for the same 4.2 MFLOP), which is what keeps shared memory and L2 below the tensor pipe.
// Warp roles per CTA: 0 = TMA producer of A, 1 = MMA issuer (the first CTA of the pair only), 2 = TMA producer of B, 3 idle,
// 4-11 = epilogue, two warps per tensor-memory quadrant, half of the tile's columns each.  Two accumulators of 256 columns (fp32:
// four of 128): the epilogue of a tile runs beside the main loop of the next.
//
// dz lives in blocks that are images of the shared-memory tiles: panels of 64 classes, in a panel one 128-byte line per
// token, the 16-byte pieces of a line permuted by the low three bits of the token as the 128-byte swizzle of tcgen05 wants
// them.  The same 8 KB of 64 tokens x 64 classes is a K-major tile for dX and an MN-major tile for dW, and every tile is one
// or two contiguous reads.
//
// fp32 operands come as three bf16 planes, x = hi + mid + lo to its 24 bits, with the exponents of fp32 and no scale: nothing in a
// tensor changes how another of its elements is held.  Six products are accumulated, the smallest first: lo*hi and hi*lo, then
// mid*mid, mid*hi and hi*mid, then hi*hi; what is dropped is below 2^-22 of |x||w|.  (Two fp16 planes under one power of two per
// tensor need three products, but one large element then costs all others their bits, and entries of dz below 2^-39 of
// the largest vanish, which is all that the classes nobody is trained on have.)  The tensor core cuts its running sum off
// toward zero at every 16-element step, an error that grows with the length of the chain, so a chain ends after 64 elements and
// the epilogue warps add the chains in registers, rounding to nearest.  The tiles are 256 x 128 (64 running sums per thread) on four
// accumulators.  A stage is one plane of both operands: eight fit, and each is free again when its products are done.
//
// Same conventions as the other tcgen05 kernels: every wait is bounded, a wait that gives up records the status and the
// kernel winds down and returns.
#include <atomic>
#include <climits>

#include "head_loss.cuh"
#include "tc_common.cuh"

namespace tbn {
namespace head {

namespace {

using namespace tc;

constexpr int kMaxStages = 24;
constexpr uint32_t kSideBytes = 128 * 128;             // one operand, one plane, one CTA: 128 rows x 64 elements
constexpr uint32_t kStageBudget = 6 * 2 * kSideBytes;  // 192 KB of stages
constexpr uint32_t kExchange = 2048;                   // per epilogue warp: 16 lines of 128 bytes
constexpr uint32_t kTmemCols = 512;
constexpr int kGroupM = 32;                            // token tiles that share a sweep over the classes
constexpr float kCoarseLse = 4096.0f;                  // |log2 of a row's sum| from which on its rounding shows in the probabilities

enum { kStats = 0, kDz = 1, kGrads = 2 };

// columns of a tile at most, and accumulators in the 512 columns of tensor memory
template <int PL> constexpr int kCols = PL == 1 ? 256 : 128;
template <int PL> constexpr int kAccs = 512 / kCols<PL>;
// epilogue warps: kGroups per tensor-memory quadrant, which share a tile's columns
constexpr int kGroups = 2, kEpiWarps = 4 * kGroups, kThreads = 128 + 32 * kEpiWarps;
template <int PL> constexpr int kWarpCols = kCols<PL> / kGroups;
// behind the stages: exchange lines, or the biases of every epilogue warp's columns
template <int MODE, int PL> constexpr uint32_t kScratch = kEpiWarps * (MODE == kGrads ? kExchange : kWarpCols<PL> * sizeof(float));

struct Control {
    uint64_t full[kMaxStages], empty[kMaxStages], d_full[4], d_empty[4];
    uint32_t tmem_base;
    int abort_flag;
};

// Two jobs at most: (0) dX and (1) dW.  The logits kernels use job 0 alone.
struct Maps { CUtensorMap a[2], b[2]; };

struct LogitsParams {
    const int32_t *n_live;                 // null: all Tpad-padded rows below n_rows, in their own order (forward)
    const RowInfo *rows;
    Labels labels;                         // without rows
    int32_t n_rows;
    int32_t bn;                            // classes of a tile: a multiple of 32 from 64 to 256
    int32_t a_rows, stages;                // token rows of a CTA's tile that are loaded; pipeline stages
    const float *bias;
    float scale2;
    int64_t Tpad;
    int32_t v0, width, w_row0;             // w_row0: w's row of class v0
    const int2 *list;                      // distillation: [T][K] (class, probability) pairs, ascending; else null
    const uint16_t *list_start;            // [T][pitch]: where the classes of each unit begin in the row's list
    int32_t K, unit, units, pitch;
    float4 *part;
    int32_t parts;
    void *dz;
    int32_t ldz;
    float *col_part;
};
struct GradParams {
    const int32_t *n_live;
    const RowInfo *rows;
    float tau;
    int64_t Tpad;
    int32_t d, v0, width, w_row0, ldz;
    int32_t want_dx, want_dw, w_panels;    // w_panels: w can be read as panels of 64 columns
    void *dx;
    float *dx_slots;
    int32_t dx_splits, dx_bf16, dx_add, dx_last;
    void *dw;
    float *dw_slots;
    int32_t dw_splits, dw_bf16, slot_ld;
};
struct KernelParams { LogitsParams l; GradParams g; int *status; };

// ---- PTX forms of the CTA pair ------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// Tells the pair's MMA warp that an accumulator has been read.  Nothing in ordinary memory goes with it (tcgen05.wait::ld and
// the tcgen05 fence order the reads), so no release at cluster scope: that waits for the thread's stores to global memory,
// about a microsecond per hand-over.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// The copy lands in this CTA; its bytes are counted on the barrier of the pair's first CTA.  Run by the whole converged warp,
// performed by the elected lane, like the MMAs: in a branch taken by one lane every operand is a per-thread value that has to
// be moved to the uniform registers first, which made the producer the slowest part of the pipeline.
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, int32_t c0, int32_t c1, int32_t c2, uint32_t bar,
                                              uint32_t leader) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %6, 0;\n\t"
        "@q cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar), "r"(leader) : "memory");
}
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, int32_t c0, int32_t c1, int32_t c2, int32_t c3,
                                              uint32_t bar, uint32_t leader) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %7, 0;\n\t"
        "@q cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar), "r"(leader) : "memory");
}
__device__ __forceinline__ void expect_tx_elect(uint32_t bar, uint32_t bytes, uint32_t leader) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %2, 0;\n\t"
        "@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes), "r"(leader) : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate,
                                         uint32_t leader) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 ad, bd;\n\t"
        "setp.ne.b32 q, %6, 0;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 ad, {%1, %3};\n\t"
        "mov.b64 bd, {%2, %3};\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f16 [%0], ad, bd, %4, p;\n\t}"
        ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
// Arrives on the barrier at this offset in both CTAs once the MMAs issued so far have completed.
__device__ __forceinline__ void commit_pair(uint32_t bar, uint32_t leader) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t.reg .b16 mask;\n\t"
        "mov.b16 mask, 3;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], mask;\n\t}"
        ::"r"(bar), "r"(leader) : "memory");
}
__device__ __forceinline__ float exp2_approx(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// ---- tile enumeration (the same arithmetic in every role) ----------------------------------------------
struct Tile {
    int job, split;
    int32_t m0, n0, bn;                    // first row of the pair's tile on either side, and its columns
    int32_t kb0, kb1;                      // 64-element steps
};

// Which tiles a CTA pair works on, in order.  The logits tiles are alike and dealt out in turn.  The gradient launch has
// two kinds: the longer ones are dealt out first, in turn; the pairs that got one fewer then take short ones alone for as
// many rounds as fit into a long one, and the rest is dealt out in turn again, beginning with those pairs.
struct Schedule {
    int32_t n_long, n_short, stride, me, shift, early, rounds, mine;
    // logits
    int32_t mt, nt, kb;
    // gradients
    int32_t long_job, nt_d, kb_job[2], splits[2], mt_job[2];

    template <int MODE, int PL>
    __device__ __forceinline__ void init(const KernelParams &p, int32_t n_live, int32_t k_logits) {
        stride = gridDim.x >> 1;
        me = blockIdx.x >> 1;
        n_short = 0; shift = 0; early = stride; rounds = 0;
        if (MODE != kGrads) {
            mt = (n_live + kTile - 1) / kTile;
            nt = (p.l.width + p.l.bn - 1) / p.l.bn;
            kb = k_logits;
            n_long = mt * nt;
            bn_logits = p.l.bn;
        } else {
            d_cols = p.g.d;
            nt_d = (p.g.d + kCols<PL> - 1) / kCols<PL>;
            mt_job[0] = p.g.want_dx ? (n_live + kTile - 1) / kTile : 0;
            mt_job[1] = p.g.want_dw ? (p.g.width + kTile - 1) / kTile : 0;
            kb_job[0] = (p.g.width + 63) / 64;
            kb_job[1] = (n_live + 63) / 64;
            splits[0] = p.g.dx_splits;
            splits[1] = p.g.dw_splits;
            const int32_t l0 = kb_job[0] / splits[0], l1 = kb_job[1] / splits[1];
            long_job = l1 > l0 ? 1 : 0;
            n_long = mt_job[long_job] * nt_d * splits[long_job];
            n_short = mt_job[long_job ^ 1] * nt_d * splits[long_job ^ 1];
            shift = n_long % stride;
            if (shift) {
                early = stride - shift;
                rounds = max(l0, l1) / max(1, min(l0, l1));
            }
        }
        mine = me < n_long ? (n_long - me + stride - 1) / stride : 0;
    }
    // The pair's step-th tile; false behind the last one.
    template <int MODE, int PL>
    __device__ __forceinline__ bool get(int32_t step, Tile &t) const {
        if (MODE != kGrads) {
            if (step >= mine) return false;
            const int32_t i = me + step * stride;
            const int32_t per_group = kGroupM * nt, g = i / per_group, rem = i - g * per_group;
            const int32_t gm = min(kGroupM, mt - g * kGroupM), n = rem / gm;
            t.job = 0; t.split = 0;
            t.m0 = (g * kGroupM + (rem - n * gm)) * kTile;
            t.n0 = n * bn_logits;
            t.bn = bn_logits;
            t.kb0 = 0; t.kb1 = kb;
            return true;
        }
        int32_t i;
        if (step < mine) {
            t.job = long_job;
            i = me + step * stride;
        } else {
            t.job = long_job ^ 1;
            const int32_t q = step - mine, pos = me >= shift ? me - shift : me - shift + stride;
            if (pos >= early) i = rounds * early + q * stride + pos;
            else i = q < rounds ? q * early + pos : rounds * early + (q - rounds) * stride + pos;
            if (i >= n_short) return false;
        }
        const int32_t row = i / nt_d;
        t.n0 = (i - row * nt_d) * kCols<PL>;
        t.bn = d_cols - t.n0 > 128 ? kCols<PL> : d_cols - t.n0 > 64 ? 128 : 64;
        t.split = row / mt_job[t.job];
        t.m0 = (row - t.split * mt_job[t.job]) * kTile;
        t.kb0 = (int32_t)((int64_t)t.split * kb_job[t.job] / splits[t.job]);
        t.kb1 = (int32_t)((int64_t)(t.split + 1) * kb_job[t.job] / splits[t.job]);
        return true;
    }
    int32_t bn_logits, d_cols;
};

// The sparse side of a row: the target class with probability 1, or the teacher's ascending list of (class, probability)
// pairs, of which the next four are kept in registers: a pair is asked for four entries before its turn, so that the entries
// of one chunk do not each cost a trip to memory.
struct Listed {
    const int2 *entry;                     // the row's list
    int32_t pos, count, next;              // next: the class of the entry at pos, INT_MAX behind the last one
    float weight;
    int2 w1, w2, w3;

    __device__ __forceinline__ int2 at(int32_t i) const { return i < count ? __ldg(entry + i) : make_int2(INT_MAX, 0); }
    __device__ __forceinline__ void begin(const LogitsParams &l, const RowInfo &r, bool live, int32_t first) {
        w1 = w2 = w3 = make_int2(INT_MAX, 0);
        pos = count = 0;
        if (l.list == nullptr) {
            entry = nullptr;
            next = live && r.label >= first ? r.label : INT_MAX;
            weight = 1.0f;
            return;
        }
        entry = l.list + (int64_t)r.row * l.K;
        count = live ? l.K : 0;
        if (count) {                                   // first entry >= first: where its unit of classes begins, or behind that
            const int32_t unit = min(first / l.unit, l.units);
            pos = (int32_t)__ldg(l.list_start + (int64_t)r.row * l.pitch + unit);
            if (unit * l.unit != first)
                while (pos < count && __ldg(&entry[pos].x) < first) ++pos;
        }
        const int2 e = at(pos);
        w1 = at(pos + 1); w2 = at(pos + 2); w3 = at(pos + 3);
        next = e.x;
        weight = __int_as_float(e.y);
    }
    __device__ __forceinline__ void step() {
        next = w1.x;
        weight = __int_as_float(w1.y);
        w1 = w2; w2 = w3;
        ++pos;
        w3 = at(pos + 3);
    }
};

__device__ __forceinline__ uint64_t f32x2_add(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// v = v * a + b, two at a time; bias: 32 floats in shared memory, 16-byte aligned, added to b where there are any
template <bool BIAS>
__device__ __forceinline__ void scale_shift(float (&v)[32], float a, float b, const float4 *bias) {
    const uint64_t a2 = f32x2_pack(a, a), b2 = f32x2_pack(b, b);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        uint64_t s0 = b2, s1 = b2;
        if (BIAS) {
            const float4 u = bias[q];
            s0 = f32x2_add(f32x2_pack(u.x, u.y), b2);
            s1 = f32x2_add(f32x2_pack(u.z, u.w), b2);
        }
        f32x2_unpack(f32x2_fma(f32x2_pack(v[4 * q], v[4 * q + 1]), a2, s0), v[4 * q], v[4 * q + 1]);
        f32x2_unpack(f32x2_fma(f32x2_pack(v[4 * q + 2], v[4 * q + 3]), a2, s1), v[4 * q + 2], v[4 * q + 3]);
    }
}
// 32 x 32 values, lane = row: returns in lane c the sum over the rows of column c (v is overwritten).
__device__ __forceinline__ float column_sums(float (&v)[32], int lane) {
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) {
        const bool upper = (lane & s) != 0;
#pragma unroll
        for (int i = 0; i < s; ++i) {
            const float send = upper ? v[i] : v[i + s], keep = upper ? v[i + s] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, s);
        }
    }
    return v[0];
}

// A lane's 32 values as the pieces [4 * upper, 4 * upper + 4) of its line of a dz panel: two whole 32-byte sectors, whose
// 16-byte halves trade places in odd lanes.  Straight from registers: through shared memory and a bulk copy the lines would
// be written in one go, but the main loop's copies and MMAs use all of shared memory's bandwidth (tiles of d = 1024 took
// 9.5 K cycles that way, against 8.2 K of MMAs).
__device__ __forceinline__ void store_line(uint16_t *line, int lane, int upper, const uint32_t (&pk)[16]) {
    const bool odd = (lane & 1) != 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t v[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = odd ? pk[8 * h + 4 + j] : pk[8 * h + j];
            v[4 + j] = odd ? pk[8 * h + j] : pk[8 * h + 4 + j];
        }
        st_global_v8(line + (((upper * 4 + 2 * h) ^ (lane & 6)) << 3), v);
    }
}
__device__ __forceinline__ uint32_t lds_b32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ void ld_global_v8(const float *ptr, float (&v)[8]) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]) : "l"(ptr) : "memory");
}
// Where a warp's rows of dX or dW go.  prev: fp32 values added first, or null; row, prev_row: this lane's row in out and prev.
// scale: what the whole sum is multiplied by, 1 for a part of it (parts of sums that are too large for fp32 would meet as
// infinities of both signs).
struct RowsOut {
    void *out;
    const float *prev;
    float scale;
    int32_t row, prev_row, ld, prev_ld, rows_in, end;      // end: the first column that is not this warp's
};
// 32 columns of every lane's row, in whole 32-byte sectors (rows a multiple of 16 elements, 32-byte aligned).  The columns
// behind end are not written, but for those of the padding of a slot's row.
__device__ __forceinline__ void write_sectors(const RowsOut &o, int lane, int32_t c0, bool out_bf16, float (&v)[32])
{
    if (lane >= o.rows_in) return;
    if (o.prev) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (c0 + 8 * q >= o.end) break;
            float w[8];
            ld_global_v8(o.prev + (int64_t)o.prev_row * o.prev_ld + c0 + 8 * q, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[8 * q + j] += w[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] *= o.scale;
    const int64_t at = (int64_t)o.row * o.ld + c0;
    if (out_bf16) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (c0 + 16 * h >= o.end) break;
            uint32_t pk[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(v[16 * h + 2 * j], v[16 * h + 2 * j + 1]);
                pk[j] = *reinterpret_cast<const uint32_t *>(&b);
            }
            st_global_v8(static_cast<__nv_bfloat16 *>(o.out) + at + 16 * h, pk);
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (c0 + 8 * q >= o.end) break;
            uint32_t u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = __float_as_uint(v[8 * q + j]);
            st_global_v8(static_cast<float *>(o.out) + at + 8 * q, u);
        }
    }
}
// Rows that are not whole sectors: through the warp's exchange lines, then a row at a time, lane = column.
__device__ __forceinline__ void write_elements(const RowsOut &o, uint32_t exchange, int lane, int32_t c0, bool out_bf16, const float (&v)[32])
{
    const int32_t c = c0 + lane;
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {             // 16 rows at a time
        if ((lane >> 4) == part) {
            const uint32_t line = exchange + (uint32_t)(lane & 15) * 128;
#pragma unroll
            for (int q = 0; q < 8; ++q)
                sts_v4(line + (uint32_t)((q ^ (lane & 7)) << 4), __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]),
                       __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
        }
        __syncwarp();
#pragma unroll 1
        for (int h = 0; h < 16; h += 8) {              // eight rows in flight
            float x[8];
            int32_t to[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int r = part * 16 + h + k;
                x[k] = __uint_as_float(lds_b32(exchange + (uint32_t)(h + k) * 128 + (uint32_t)(((lane >> 2) ^ k) << 4) + (lane & 3) * 4));
                to[k] = __shfl_sync(0xffffffffu, o.row, r);
                if (o.prev) {
                    const int32_t from = __shfl_sync(0xffffffffu, o.prev_row, r);
                    if (r < o.rows_in && c < o.end) x[k] += o.prev[(int64_t)from * o.prev_ld + c];
                }
                x[k] *= o.scale;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (part * 16 + h + k < o.rows_in && c < o.end) {
                    const int64_t at = (int64_t)to[k] * o.ld + c;
                    if (out_bf16) static_cast<__nv_bfloat16 *>(o.out)[at] = __float2bfloat16_rn(x[k]);
                    else static_cast<float *>(o.out)[at] = x[k];
                }
            }
        }
        __syncwarp();
    }
}

// ---- the kernel ------------------------------------------------------------------------------------------
template <int MODE, int PL, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1) __cluster_dims__(2, 1, 1)
head_kernel(const __grid_constant__ Maps maps, const __grid_constant__ KernelParams p, const int32_t k_logits)
{
    static_assert(PL == 1 || PL == 3, "bf16, or the three parts of fp32");
    constexpr uint32_t kBBytes = kCols<PL> * 64;       // B of a gradient tile: one plane, one CTA
    constexpr int kFewStages = kStageBudget / (kSideBytes + kBBytes);
    // instruction descriptor: D fp32, A and B bf16, M = 256, N added per tile; bits 15 / 16 select the MN-major form of A / B
    constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kTile >> 4) << 24);
    // 128-byte swizzle, 8-row groups 1024 bytes apart, descriptor version 1
    constexpr uint32_t kDescHi = 64u | (1u << 14) | (2u << 29);

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t pad = (1024u - (raw & 1023u)) & 1023u;
    const uint32_t stage0 = raw + pad;
    Control *ctl = reinterpret_cast<Control *>(smem_raw + pad + kStageBudget + kScratch<MODE, PL>);
    volatile int *abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int detail = (int)(blockIdx.x & 0xffff);

    if (MODE == kDz) pdl_launch_dependents();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kMaxStages; ++s) { mbar_init(smem_u32(&ctl->full[s]), 1); mbar_init(smem_u32(&ctl->empty[s]), 1); }
        for (int s = 0; s < kAccs<PL>; ++s) { mbar_init(smem_u32(&ctl->d_full[s]), 1); mbar_init(smem_u32(&ctl->d_empty[s]), 2 * kEpiWarps); }
        ctl->abort_flag = 0;
        fence_barrier_init();
        fence_proxy_async();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = ctl->tmem_base;
    pdl_wait();

    const int32_t n_live = MODE == kGrads ? *p.g.n_live : p.l.n_live ? *p.l.n_live : p.l.n_rows;
    Schedule sched = {};
    sched.init<MODE, PL>(p, n_live, k_logits);
    Tile t;
    bool ok = true;
    // A logits stage holds the rows that exist: with few tokens most of it is classes, and more stages fit.  (The MMAs read
    // 128 token rows all the same; what lies behind the loaded ones belongs to later parts of the pipeline and only
    // reaches the accumulator rows of tokens that do not exist.)
    const uint32_t a_bytes = MODE == kGrads ? kSideBytes : (uint32_t)p.l.a_rows * 128;
    const uint32_t b_bytes = MODE == kGrads ? kBBytes : (uint32_t)p.l.bn * 64;
    const uint32_t stage_bytes = a_bytes + b_bytes;    // one plane
    const uint32_t n_stages = MODE == kGrads ? kFewStages : (uint32_t)p.l.stages;

    if (warp == 0 || warp == 2) {
        // ---------------- TMA producers: warp 0 brings A, warp 2 brings B ----------------
        const bool is_a = warp == 0;
        const uint32_t leader = elect_one();
        const uint32_t full0 = __shfl_sync(0xffffffffu, smem_u32(&ctl->full[0]), 0), bar0 = map_to_rank(full0, 0);
        const uint32_t sm0 = __shfl_sync(0xffffffffu, stage0, 0);
        Pipe px;
        for (int32_t step = 0; ok && sched.get<MODE, PL>(step, t); ++step) {
            const int32_t r0 = is_a ? t.m0 + (int32_t)rank * 128 : t.n0 + (int32_t)rank * (t.bn / 2);
            const int job = __shfl_sync(0xffffffffu, t.job, 0);
            const CUtensorMap *map = is_a ? &maps.a[job] : &maps.b[job];
            // A half tile of rows that do not exist is not loaded: what the second CTA holds instead reaches no result
            const bool second = t.m0 + 128 < (job == 0 ? n_live : p.g.width), load_a = rank == 0 || second;
            for (int32_t kb = t.kb0; ok && kb < t.kb1; ++kb) {
#pragma unroll
                for (int u = 0; u < PL; ++u) {
                    const int pl = PL == 1 ? 0 : u == 0 ? 2 : u - 1;             // lo, hi, mid: in the order of their first use
                    ok = wait_bar(smem_u32(&ctl->empty[px.stage]), px.phase ^ 1u, abort_flag, p.status, (40 << 24) | (px.stage << 16) | detail);
                    if (!ok) break;
                    const uint32_t bar = bar0 + px.stage * 8, sa = sm0 + px.stage * stage_bytes, sb = sa + a_bytes;
                    if (is_a && rank == 0) expect_tx_elect(full0 + px.stage * 8, (second ? 2 : 1) * a_bytes + 2 * b_bytes, leader);
                    if (MODE != kGrads) {
                        if (!is_a) tma_load_pair(sb, map, kb * 64, p.l.w_row0 + r0, pl, bar, leader);
                        else if (load_a) tma_load_pair(sa, map, kb * 64, r0, pl, bar, leader);
                    } else {
                        // dX: dz as 128 tokens x 64 classes, dW: as two panels of 64 tokens x 64 classes
                        const int32_t krow = (job == 0 ? p.g.w_row0 : 0) + kb * 64;
                        if (is_a) {
                            if (!load_a) {}
                            else if (job == 0) tma_load_pair(sa, map, 0, r0, kb, pl, bar, leader);
                            else tma_load_pair(sa, map, 0, kb * 64, r0 / 64, pl, bar, leader);
                        } else if (job == 1 || p.g.w_panels) {
                            tma_load_pair(sb, map, r0 & 63, krow, r0 >> 6, pl, bar, leader);
                        } else {                       // rows that are not whole panels
                            tma_load_pair(sb, map, r0, krow, pl, bar, leader);
                            tma_load_pair(sb + kSideBytes / 2, map, r0 + 64, krow, pl, bar, leader);
                        }
                    }
                    px.advance(n_stages);
                }
            }
        }
        if (!ok) {                                     // let copies in flight land before the shared memory goes away
            const uint64_t t0 = global_timer_ns();
            while (global_timer_ns() - t0 < 20000000ull) {}
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer: the whole warp runs the loop, one elected lane issues ----------------
        if (rank == 0) {
            const uint32_t tmem_u = __shfl_sync(0xffffffffu, tmem_base, 0);
            const uint32_t leader = elect_one();
            Pipe px, pd;
            for (int32_t step = 0; ok && sched.get<MODE, PL>(step, t); ++step) {
                if (PL == 1) {
                    ok = wait_bar(smem_u32(&ctl->d_empty[pd.stage]), pd.phase ^ 1u, abort_flag, p.status, (41 << 24) | detail);
                    if (!ok) break;
                }
                const bool a_mn = MODE == kGrads && t.job == 1, b_mn = MODE == kGrads;
                const uint32_t idesc = kIdesc | ((uint32_t)(t.bn >> 3) << 17) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
                // low descriptor word: start address in 16-byte units, leading offset (between 64-element panels of the
                // MN-major form: 8192 bytes).  A step of 16 along K: 32 bytes inside the swizzled row, or two 8-row groups.
                const uint32_t a_hi = (a_mn ? 512u : 1u) << 16, b_hi = (b_mn ? 512u : 1u) << 16;
                const uint32_t a_step = a_mn ? 128u : 2u, b_step = b_mn ? 128u : 2u;
                if constexpr (PL == 1) {
                    const uint32_t d_addr = tmem_u + pd.stage * kCols<PL>;
                    for (int32_t kb = t.kb0; kb < t.kb1; ++kb) {
                        ok = wait_bar(smem_u32(&ctl->full[px.stage]), px.phase, abort_flag, p.status, (42 << 24) | (px.stage << 16) | detail);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t sa = stage0 + px.stage * stage_bytes, sb = sa + a_bytes;
                        const uint32_t a_lo = ((sa & 0x3FFFFu) >> 4) | a_hi, b_lo = ((sb & 0x3FFFFu) >> 4) | b_hi;
#pragma unroll
                        for (int st = 0; st < 4; ++st)
                            mma_pair(d_addr, a_lo + st * a_step, b_lo + st * b_step, kDescHi, idesc, st > 0 ? 1u : (uint32_t)(kb > t.kb0), leader);
                        commit_pair(smem_u32(&ctl->empty[px.stage]), leader);
                        px.advance(n_stages);
                    }
                } else {
                    // the products of part i of A and part j of B: four MMAs
                    auto product = [&](uint32_t d_addr, const Pipe &a, const Pipe &b, uint32_t accumulate) {
                        const uint32_t sa = stage0 + a.stage * stage_bytes, sb = stage0 + b.stage * stage_bytes + a_bytes;
                        const uint32_t a_lo = ((sa & 0x3FFFFu) >> 4) | a_hi, b_lo = ((sb & 0x3FFFFu) >> 4) | b_hi;
#pragma unroll
                        for (int st = 0; st < 4; ++st)
                            mma_pair(d_addr, a_lo + st * a_step, b_lo + st * b_step, kDescHi, idesc, st > 0 ? 1u : accumulate, leader);
                    };
                    auto loaded = [&](const Pipe &s) {
                        return wait_bar(smem_u32(&ctl->full[s.stage]), s.phase, abort_flag, p.status, (42 << 24) | (s.stage << 16) | detail);
                    };
                    for (int32_t kb = t.kb0; kb < t.kb1; ++kb) {                 // one chain: 64 elements
                        ok = wait_bar(smem_u32(&ctl->d_empty[pd.stage]), pd.phase ^ 1u, abort_flag, p.status, (41 << 24) | detail);
                        if (!ok) break;
                        const uint32_t d_addr = tmem_u + pd.stage * kCols<PL>;
                        Pipe lo = px;
                        px.advance(n_stages);
                        Pipe hi = px;
                        px.advance(n_stages);
                        Pipe mid = px;
                        px.advance(n_stages);
                        ok = loaded(lo) && loaded(hi);
                        if (!ok) break;
                        tc_fence_after();
                        product(d_addr, lo, hi, 0u);
                        product(d_addr, hi, lo, 1u);
                        commit_pair(smem_u32(&ctl->empty[lo.stage]), leader);
                        ok = loaded(mid);
                        if (!ok) break;
                        tc_fence_after();
                        product(d_addr, mid, mid, 1u);
                        product(d_addr, mid, hi, 1u);
                        product(d_addr, hi, mid, 1u);
                        commit_pair(smem_u32(&ctl->empty[mid.stage]), leader);
                        product(d_addr, hi, hi, 1u);
                        commit_pair(smem_u32(&ctl->empty[hi.stage]), leader);
                        commit_pair(smem_u32(&ctl->d_full[pd.stage]), leader);
                        pd.advance(kAccs<PL>);
                    }
                }
                if (!ok) break;
                if (PL == 1) {
                    commit_pair(smem_u32(&ctl->d_full[pd.stage]), leader);
                    pd.advance(kAccs<PL>);
                }
            }
            if (!ok) {                                 // no MMA may still read shared or tensor memory when they go away
                const uint64_t t0 = global_timer_ns();
                while (global_timer_ns() - t0 < 20000000ull) {}
            }
        }
        __syncwarp();
    } else if (warp >= 4) {
        // ---------------- epilogue: thread = row, a group's share of the tile's columns in chunks of 32 --------
        const int ew = warp - 4, qd = warp & 3, group = ew >> 2;
        const uint32_t t_lane = tmem_base + ((uint32_t)(qd * 32) << 16);
        const uint32_t exchange = stage0 + kStageBudget + (uint32_t)ew * kExchange;
        Pipe pd;
        const float sc = MODE != kGrads ? p.l.scale2 : 1.0f;
        const float mantissa = PL == 1 && MODE != kStats ? common_mantissa(MODE == kDz ? p.l.rows : p.g.rows, n_live) : 1.0f;
        // what a tile needs to know about this lane's row, asked for while the tile before it is worked on
        auto row_info = [&](const Tile &u) {
            RowInfo r = {0.0f, 0.0f, -1, 0};
            const int32_t at = u.m0 + (int32_t)rank * 128 + qd * 32 + lane;
            if (at >= n_live) return r;
            if (MODE == kGrads) {
                if (u.job == 0) r.row = p.g.rows[at].row;
            } else if (p.l.rows) {
                r = p.l.rows[at];
            } else {
                r.row = at;
                if (!p.l.labels.flags && p.l.labels.live(at)) r.label = (int32_t)p.l.labels.target[at];
            }
            return r;
        };
        Tile next;
        bool more = sched.get<MODE, PL>(0, next);
        RowInfo next_info = {0.0f, 0.0f, -1, 0};
        if (more) next_info = row_info(next);
        for (int32_t step = 0; more; ++step) {
            t = next;
            const RowInfo info = next_info;
            const int32_t row0 = t.m0 + (int32_t)rank * 128 + qd * 32, row = row0 + lane;
            const int32_t hc = t.bn / kGroups, col0 = t.n0 + group * hc;
            const bool live = row < n_live;
            // rows that nothing is written for: dz has zeros up to the next 64 tokens, which dW contracts over
            const int32_t row_end = MODE == kDz ? (n_live + 63) & ~63 : MODE == kGrads && t.job == 1 ? p.g.width : n_live;
            const int chunks = row0 < row_end ? kWarpCols<PL> / 32 : 0;
            Listed list;
            if (MODE != kGrads) list.begin(p.l, info, live, p.l.v0 + col0);
            float *bias_s = reinterpret_cast<float *>(smem_raw + pad + kStageBudget) + ew * kWarpCols<PL>;
            if (BIAS) {                                // times log2(e) / tau, finite ones kept finite; -infinity behind the last class
#pragma unroll
                for (int j = 0; j < kWarpCols<PL> / 32; ++j) {
                    const int32_t c = col0 + j * 32 + lane;
                    const float b = j * 32 < hc && c < p.l.width ? __ldg(p.l.bias + p.l.v0 + c) : -INFINITY;
                    bias_s[j * 32 + lane] = b == -INFINITY ? b : fmaxf(b * p.l.scale2, -3.402823466e38f) + (b - b);
                }
                __syncwarp();
            }
            more = sched.get<MODE, PL>(step + 1, next);
            if (more) next_info = row_info(next);
            // the tile's sums: left in tensor memory, or (three planes) added up from its 64-element chains in registers
            float acc[PL == 3 ? 64 : 1];
            uint32_t t_acc = 0;
            if constexpr (PL == 1) {
                ok = wait_bar(smem_u32(&ctl->d_full[pd.stage]), pd.phase, abort_flag, p.status, (43 << 24) | detail);
                if (!ok) break;
                tc_fence_after();
                t_acc = t_lane + pd.stage * kCols<PL> + (uint32_t)(group * hc);
            } else {
#pragma unroll
                for (int j = 0; j < 64; ++j) acc[j] = 0.0f;
                for (int32_t kb = t.kb0; kb < t.kb1; ++kb) {
                    ok = wait_bar(smem_u32(&ctl->d_full[pd.stage]), pd.phase, abort_flag, p.status, (43 << 24) | detail);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t t_sum = t_lane + pd.stage * kCols<PL> + (uint32_t)(group * hc);
                    if (chunks) {
                        uint32_t r[32], r2[32];        // of a narrow tile, up to 32 columns behind its own are read and not used
                        tmem_ld_32x32(t_sum, r);
                        tmem_ld_32x32(t_sum + 32, r2);
                        tc_wait_ld();
#pragma unroll
                        for (int j = 0; j < 32; ++j) { acc[j] += __uint_as_float(r[j]); acc[32 + j] += __uint_as_float(r2[j]); }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(map_to_rank(smem_u32(&ctl->d_empty[pd.stage]), 0));
                    pd.advance(kAccs<PL>);
                }
                if (!ok) break;
            }
            // 32 columns of the tile.  One plane: the next 32 are asked for before these are worked on.
            uint32_t ahead[PL == 1 ? 32 : 1];
            if constexpr (PL == 1) { if (chunks) tmem_ld_32x32(t_acc, ahead); }
            auto load_chunk = [&](int ch, float (&out)[32]) {
                if constexpr (PL == 1) {
                    tc_wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; ++j) out[j] = __uint_as_float(ahead[j]);
                    if ((ch + 1) * 32 < hc) tmem_ld_32x32(t_acc + (ch + 1) * 32, ahead);
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) out[j] = ch == 0 ? acc[j] : acc[32 + j];
                }
            };

            if (MODE == kStats) {
                float m = -INFINITY, l = 0.0f, dot = 0.0f;     // m: without a bias before scaling
#pragma unroll 1
                for (int ch = 0; ch < chunks; ++ch) {
                    if (ch * 32 >= hc) continue;
                    const int32_t c0 = col0 + ch * 32, end = min(c0 + 32, min(col0 + hc, p.l.width));
                    float v[32];
                    load_chunk(ch, v);
                    if (BIAS) scale_shift<true>(v, sc, 0.0f, reinterpret_cast<const float4 *>(bias_s + ch * 32));
                    if (c0 + 32 > end) {               // behind the last class, or the other warps' columns
#pragma unroll
                        for (int j = 0; j < 32; ++j) if (c0 + j >= end) v[j] = -INFINITY;
                    }
                    const float vs = BIAS ? 1.0f : sc;
                    while (list.next < p.l.v0 + end) {
                        const int rel = list.next - (p.l.v0 + c0);
                        float z = 0.0f;
#pragma unroll
                        for (int j = 0; j < 32; ++j) z = rel == j ? v[j] : z;
                        if (list.weight != 0.0f) dot = fmaf(list.weight, z * vs, dot);     // 0 times a class at -infinity is 0
                        list.step();
                    }
                    __syncwarp();
                    float mx[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
                    for (int j = 4; j < 32; ++j) mx[j & 3] = fmaxf(mx[j & 3], v[j]);
                    // The difference to the maximum before it is scaled: exact near the maximum, so that the largest term is 1
                    // however large the logits are (scaled first, a product and its rounded self differ by more than exp2's range
                    // from 2^31 on: infinite sums)
                    const float m_new = fmaxf(m, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
                    const float ref = m_new == -INFINITY ? 0.0f : m_new;
                    const uint64_t ref2 = f32x2_pack(-ref, -ref), vs2 = f32x2_pack(vs, vs);
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        uint64_t u = f32x2_add(f32x2_pack(v[j], v[j + 1]), ref2);
                        if (!BIAS) u = f32x2_mul(u, vs2);
                        f32x2_unpack(u, v[j], v[j + 1]);
                    }
                    uint64_t s0 = 0, s1 = 0;           // four running sums
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        s0 = f32x2_add(s0, f32x2_pack(exp2_approx(v[j]), exp2_approx(v[j + 1])));
                        s1 = f32x2_add(s1, f32x2_pack(exp2_approx(v[j + 2]), exp2_approx(v[j + 3])));
                    }
                    float e0, e1;
                    f32x2_unpack(f32x2_add(s0, s1), e0, e1);
                    l = l * exp2_approx((m - ref) * vs) + (e0 + e1);
                    m = m_new;
                }
                if (live) {
                    p.l.part[(int64_t)row * p.l.parts + (p.l.v0 + col0) / hc] = make_float4(BIAS ? m : m * sc, l, dot, 0.0f);
                }
            } else if (MODE == kDz) {
                const bool all_live = __all_sync(0xffffffffu, live);
                const float row_g = PL == 1 ? info.g / mantissa : info.g;
                // lse is a float: a logit and the lse that it makes up differ by up to 2^-22 of it (four roundings).  Where that is
                // more than a thousandth, what comes within it, and what comes out above lse, is a probability of 1.
                const bool coarse = fabsf(info.lse2) > kCoarseLse;
                const bool any_coarse = __any_sync(0xffffffffu, coarse);
                const float lse2 = coarse ? info.lse2 - 1.5f * 0x1p-22f * fabsf(info.lse2) : info.lse2;
                const int32_t panels = p.l.ldz / 64;
                uint16_t *dz = static_cast<uint16_t *>(p.l.dz);
#pragma unroll 1
                for (int ch = 0; ch < chunks; ++ch) {
                    const int32_t c0 = col0 + ch * 32;
                    if (ch * 32 >= hc || c0 >= p.l.ldz) continue;
                    float v[32];
                    load_chunk(ch, v);
                    scale_shift<BIAS>(v, sc, -lse2, reinterpret_cast<const float4 *>(bias_s + ch * 32));
                    if (any_coarse) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = coarse && v[j] > 0.0f ? 0.0f : v[j];       // NaN stays
                    }
                    if (!BIAS && c0 + 32 > p.l.width) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) if (c0 + j >= p.l.width) v[j] = -INFINITY;
                    }
                    const uint64_t g2 = f32x2_pack(row_g, row_g);
#pragma unroll
                    for (int j = 0; j < 32; j += 2)
                        f32x2_unpack(f32x2_mul(f32x2_pack(exp2_approx(v[j]), exp2_approx(v[j + 1])), g2), v[j], v[j + 1]);
                    while (list.next < p.l.v0 + c0 + 32) {
                        const int rel = list.next - (p.l.v0 + c0);
                        const float sub = row_g * list.weight;
#pragma unroll
                        for (int j = 0; j < 32; ++j) if (rel == j) v[j] -= sub;
                        list.step();
                    }
                    __syncwarp();
                    if (!all_live) {                   // rows behind the last kept token: exact zeros, whatever was staged
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = live ? v[j] : 0.0f;
                    }
                    uint16_t *dst = dz + ((int64_t)(c0 >> 6) * p.l.Tpad + row) * 64;
                    if (p.l.col_part) {
                        float sum[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum[j] = v[j];
                        const float s = column_sums(sum, lane);
                        p.l.col_part[(int64_t)(row >> 5) * p.l.ldz + c0 + lane] = s;
                    }
#pragma unroll
                    for (int pl = 0; pl < PL; ++pl) {  // the parts of fp32: each of what the ones before leave over
                        uint32_t pk[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                            pk[i] = *reinterpret_cast<const uint32_t *>(&h);
                            if (pl + 1 < PL) {
                                const float2 back = __bfloat1622float2(h);
                                v[2 * i] -= back.x;
                                v[2 * i + 1] -= back.y;
                            }
                        }
                        store_line(dst + (int64_t)pl * panels * p.l.Tpad * 64, lane, (c0 >> 5) & 1, pk);
                    }
                }
            } else {
                // A lane stores its own row in whole 32-byte sectors: 32 lines per instruction, so the load / store unit, one
                // line per cycle, needs 2 K cycles for a bf16 tile.  (16-byte stores took 10 K; passing the values through
                // shared memory for stores along the rows 5 K, most of it latency.)
                const GradParams &g = p.g;
                const bool empty = t.kb0 >= t.kb1;     // nothing was contracted: the accumulator holds no result
                const bool is_dx = t.job == 0;
                const int32_t rows_in = (is_dx ? n_live : g.width) - row0;             // rows of this warp that exist
                const int splits = is_dx ? g.dx_splits : g.dw_splits;
                float *slot = is_dx ? g.dx_slots : g.dw_slots;
                if (slot) slot += ((int64_t)t.split * (is_dx ? g.Tpad : round_up64(g.width, kTile)) + row0) * g.slot_ld;
                const bool to_slot = slot != nullptr && (splits > 1 || !(is_dx && g.dx_last));
                RowsOut o;
                o.out = to_slot ? static_cast<void *>(slot) : is_dx ? g.dx : g.dw;
                o.row = to_slot ? lane : is_dx ? info.row : g.v0 + row0 + lane;
                o.prev = !(is_dx && g.dx_add) ? nullptr : slot ? slot : static_cast<const float *>(g.dx);
                o.prev_row = slot ? lane : info.row;
                o.ld = to_slot ? g.slot_ld : g.d;
                o.prev_ld = slot ? g.slot_ld : g.d;
                o.scale = to_slot || (is_dx && !g.dx_last) ? 1.0f : g.tau * mantissa;
                o.rows_in = rows_in; o.end = min(to_slot ? g.slot_ld : g.d, col0 + hc);
                const bool out_bf16 = !to_slot && (is_dx ? g.dx_bf16 : g.dw_bf16);
                const bool sectors = o.ld % 16 == 0 && (!o.prev || o.prev_ld % 16 == 0) &&
                                     ((reinterpret_cast<uintptr_t>(o.out) | reinterpret_cast<uintptr_t>(o.prev)) & 31) == 0;
#pragma unroll 1
                for (int ch = 0; ch < chunks; ++ch) {
                    const int32_t c0 = col0 + ch * 32;
                    if (ch * 32 >= hc || c0 >= g.d) continue;
                    float v[32];
                    load_chunk(ch, v);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = empty ? 0.0f : v[j];
                    if (sectors) write_sectors(o, lane, c0, out_bf16, v);
                    else write_elements(o, exchange, lane, c0, out_bf16, v);
                    __syncwarp();
                }
            }
            __syncwarp();
            if (PL == 1) {
                tc_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_rank(smem_u32(&ctl->d_empty[pd.stage]), 0));
                pd.advance(kAccs<PL>);
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    // The small kernels that follow the other two kinds are placed now, all over the GPU, rather than on the first SMs to become
    // free (join 4.3 -> 3.0 us, sums of the splits 4.9 -> 3.2 us); the gradient launch that follows dz needs a whole SM anyway.
    if (MODE != kDz) pdl_launch_dependents();
    cluster_sync();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
    }
}

// ---- host side -----------------------------------------------------------------------------------------
// 64 x box_rows boxes of an operand's planes; what lies outside is read as zero.
bool make_map(CUtensorMap *map, const void *data, int32_t cols, int64_t rows, int64_t planes, int32_t ld, int64_t plane_rows, int box_rows)
{
    EncodeTiledFn encode = encode_tiled_fn();
    if (!encode) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)plane_rows * ld * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(data), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Panels of 64 columns, `box_panels` of them (64 x box_rows each) per copy.  The rows are whole panels (ld % 64 == 0).
bool make_panel_map(CUtensorMap *map, const void *data, int64_t rows, int64_t row_bytes, int64_t panels, int64_t panel_bytes, int64_t planes,
                    int64_t plane_bytes, int box_rows, int box_panels, CUtensorMapSwizzle swizzle)
{
    EncodeTiledFn encode = encode_tiled_fn();
    if (!encode) return false;
    const cuuint64_t dims[4] = {64, (cuuint64_t)rows, (cuuint64_t)panels, (cuuint64_t)planes};
    const cuuint64_t strides[3] = {(cuuint64_t)row_bytes, (cuuint64_t)panel_bytes, (cuuint64_t)plane_bytes};
    const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, (cuuint32_t)box_panels, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(data), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MODE, int PL, bool BIAS>
int launch(const Maps &maps, const KernelParams &p, int64_t tiles, int32_t k_logits, cudaStream_t s)
{
    const int pairs = sm_count() / 2;
    if (pairs <= 0) return TBN_ERR_CUDA;
    if (tiles <= 0) return TBN_OK;
    constexpr size_t smem = kStageBudget + kScratch<MODE, PL> + sizeof(Control) + 1024;
    static_assert(smem <= 227 * 1024, "shared memory");
    auto kern = head_kernel<MODE, PL, BIAS>;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return TBN_ERR_CUDA;
    static std::atomic<bool> ready[64];                // the attribute is per device; setting it twice is harmless
    if (!ready[dev].load(std::memory_order_acquire)) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return TBN_ERR_CUDA;
        ready[dev].store(true, std::memory_order_release);
    }
    const unsigned grid = 2u * (unsigned)(tiles < pairs ? tiles : pairs);
    return launch_pdl(kern, dim3(grid), dim3(kThreads), smem, s, maps, p, k_logits) == cudaSuccess ? TBN_OK : TBN_ERR_CUDA;
}

template <int MODE>
int launch_logits(const LogitsArgs &a, cudaStream_t s)
{
    Maps maps = {};
    const int64_t rows = a.T < 128 ? (a.T + 7) / 8 * 8 : 128;
    if (!make_map(&maps.a[0], a.x.data, a.x.cols, a.x.rows, a.planes, a.x.ld, a.x.plane_rows, (int)rows) ||
        !make_map(&maps.b[0], a.w.data, a.w.cols, a.w.rows, a.planes, a.w.ld, a.w.plane_rows, a.bn / 2))
        return TBN_ERR_CUDA;
    KernelParams p = {};
    LogitsParams &l = p.l;
    l.n_live = a.n_live; l.rows = a.rows; l.labels = a.labels; l.n_rows = (int32_t)a.T; l.bn = a.bn;
    l.a_rows = (int32_t)rows;
    const int64_t stage = rows * 128 + a.bn * 64, fit = (kStageBudget - kSideBytes + rows * 128) / stage;
    l.stages = (int32_t)(fit > kMaxStages ? kMaxStages : fit);
    l.bias = a.bias; l.scale2 = a.scale2; l.Tpad = a.Tpad; l.v0 = a.v0; l.width = a.width; l.w_row0 = a.w_row0;
    l.list = a.list; l.list_start = a.list_start; l.K = a.K; l.unit = a.unit; l.units = a.units; l.pitch = a.pitch;
    l.part = a.part; l.parts = a.parts;
    l.dz = a.dz; l.ldz = a.ldz; l.col_part = a.col_part;
    p.status = a.status;
    const int64_t tiles = (a.T + kTile - 1) / kTile * ((a.width + a.bn - 1) / a.bn);
    if (tiles > INT_MAX) return TBN_ERR_UNSUPPORTED;
    const int32_t kb = (a.x.cols + 63) / 64;
    if (a.planes == 1) return a.bias ? launch<MODE, 1, true>(maps, p, tiles, kb, s) : launch<MODE, 1, false>(maps, p, tiles, kb, s);
    return a.bias ? launch<MODE, 3, true>(maps, p, tiles, kb, s) : launch<MODE, 3, false>(maps, p, tiles, kb, s);
}

}  // namespace

// Streaming multiprocessors of the current device, 0 on error.
int sm_count()
{
    static std::atomic<int> cache[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    int n = cache[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
        cache[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

int launch_head_stats(const LogitsArgs &a, cudaStream_t s) { return launch_logits<kStats>(a, s); }
int launch_head_dz(const LogitsArgs &a, cudaStream_t s) { return launch_logits<kDz>(a, s); }

int launch_head_grads(const GradArgs &a, cudaStream_t s)
{
    Maps maps = {};
    // dz is written up to the next multiple of 64 tokens, with zeros behind the last kept one: that is what dW contracts over.  The
    // lines behind that hold anything; dX loads them with its 128 tokens, into accumulator rows that are not stored.
    const int64_t dz_panels = a.ldz / 64, dz_panel = a.Tpad * 128;
    const bool w_panels = a.w.ld % 64 == 0;
    auto by_panels = [&a](CUtensorMap *m, const Operand &o) {
        return make_panel_map(m, o.data, o.rows, (int64_t)o.ld * 2, o.ld / 64, 128, a.planes, o.plane_rows * o.ld * 2, 64,
                              a.planes == 1 ? 2 : 1, CU_TENSOR_MAP_SWIZZLE_128B);
    };
    if (!make_panel_map(&maps.a[0], a.dz, a.Tpad, 128, dz_panels, dz_panel, a.planes, dz_panels * dz_panel, 128, 1, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !make_panel_map(&maps.a[1], a.dz, a.Tpad, 128, dz_panels, dz_panel, a.planes, dz_panels * dz_panel, 64, 2, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !(w_panels ? by_panels(&maps.b[0], a.w) : make_map(&maps.b[0], a.w.data, a.w.cols, a.w.rows, a.planes, a.w.ld, a.w.plane_rows, 64)) ||
        !by_panels(&maps.b[1], a.x))
        return TBN_ERR_CUDA;
    KernelParams p = {};
    GradParams &g = p.g;
    g.n_live = a.n_live; g.rows = a.rows; g.tau = a.tau; g.Tpad = a.Tpad; g.d = a.d; g.v0 = a.v0; g.width = a.width; g.w_row0 = a.w_row0; g.ldz = a.ldz;
    g.want_dx = a.want_dx; g.want_dw = a.want_dw; g.w_panels = w_panels;
    g.dx = a.dx; g.dx_slots = a.dx_slots; g.dx_splits = a.dx_splits; g.dx_bf16 = a.dx_bf16; g.dx_add = a.dx_add; g.dx_last = a.dx_last;
    g.dw = a.dw; g.slot_ld = a.slot_ld; g.dw_slots = a.dw_slots; g.dw_splits = a.dw_splits; g.dw_bf16 = a.dw_bf16;
    p.status = a.status;
    const int64_t cols = a.planes == 1 ? kCols<1> : kCols<3>, nt = (a.d + cols - 1) / cols;
    const int64_t tiles = (a.want_dx ? (a.T + kTile - 1) / kTile * nt * a.dx_splits : 0) +
                          (a.want_dw ? (a.width + kTile - 1) / kTile * nt * a.dw_splits : 0);
    if (tiles > INT_MAX) return TBN_ERR_UNSUPPORTED;
    return a.planes == 1 ? launch<kGrads, 1, false>(maps, p, tiles, 0, s) : launch<kGrads, 3, false>(maps, p, tiles, 0, s);
}

}  // namespace head
}  // namespace tbn
