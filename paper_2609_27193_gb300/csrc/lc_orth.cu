// lc_orth.cu -- an update of a weight matrix made nearly orthogonal by
// Newton-Schulz products: X = U / (|U| + eps), and `steps` times
//
//   A = X X^T,   X <- a X + (b A + c A^2) X
//
// over the shorter side (a matrix with more rows than columns is worked on
// transposed).  Each step takes a singular value s to a s + b s^3 + c s^5.
//
// The products are on the 5th-generation tensor cores, fp16 operands and fp32 sums:
//
//   * The state X is kept in fp32 beside its operand.  (With the fp16 number as state a matrix
//     of 8 directions over noise of 1e-4 came out 4e-2 off, so 6e-4; with bf16 3e-1.)
//   * The diagonals of A and of B = b A + c A^2 are far larger than the rest and stay in fp32, beside
//     the operands: A^2 = A0^2 + (d_i + d_j) A0 + d^2, and X's row i is multiplied by a + e_i.  That
//     takes the error from 1.7e-3 to 5e-4 (256 x 1024), below the output's rounding of 1.7e-3.
//   * Operands are scaled by powers of two.  No element of X, A or B is larger than the matrix's
//     largest singular value, which the coefficients bound, so nothing overflows fp16.
//   * A and B are symmetric: the tiles on and above the diagonal are computed, and a product reads the
//     others as transposes of those, which the tensor core takes either way.
//
// Matrices of up to 128 rows (of the shorter side) and 4096 columns stay in the memory of one cluster, one
// launch (orth_small_kernel).  Others take three: one moves the momentum and leaves sums of squares, one
// writes X in the products' layout, one does all products.  (256 x 256: 4, 5 and 63 us, 76 among others.)
//
// Matrices lie in the workspace in boxes of 64 x 64, rows of 128 bytes swizzled as the operands are
// in shared memory: one bulk tensor copy brings two boxes, above or beside one another, and the same box
// serves with its rows along the reduction or across it.
//
// The product kernel is one cooperative launch: its CTAs go through the 3 * steps
// products together, with a barrier of the whole grid between them (1.5 us; 15 launches would keep
// the host busy for 40).  Two CTAs of a cluster share tiles of 256 x 256 or 256 x 128 (PAIR), or a CTA has
// one of 128 x 64.  Warp 0 brings the operands, warp 1 issues the products into two accumulators in turn,
// warps 4-19 turn the finished one into the next operand.  Large products run at the tensor cores' power
// limit (4096 x 14336: 0.30 to 0.36 us for 256 x 256 x 64 on a pair, where a cuBLAS product of 8192 takes 0.32 to
// 0.36); small ones are 15 times the latency of copies (0.8 us), accumulator (1) and barrier (1.5).
//
// Waits are bounded.  A copying or issuing warp whose wait ran out stops, so the accumulator that the summing warps wait
// for does not come: their own wait runs out, the CTA's outputs are NaN, and with the next barrier everybody's.
#include <cuda.h>
#include <cuda_fp16.h>

#include <cmath>

#include "lc_bulk.cuh"
#include "lc_ops.cuh"

namespace lc {
namespace {

constexpr int kBox = 64;                    // rows and columns of a box
constexpr int kBoxBytes = kBox * kBox * 2;
constexpr int kCtaRows = 128;               // rows of the left operand in a CTA
constexpr int kSumWarp = 4, kSumWarps = 16; // the first (a multiple of 4) of the warps that read the accumulators, and their number
constexpr int kThreads = (kSumWarp + kSumWarps) * 32;
constexpr int kChunk = 16;                  // columns that such a warp works on at a time
constexpr int kMaxSteps = 16;
constexpr int kNormCtas = 1216;              // most partial sums of squares of a matrix

// A tile is of one CTA, 128 x 64, or of a pair of them with half of the rows each, 256 x 256 or 256 x 128 (kRows x up to
// kCols).
template <bool PAIR>
struct TileOf {
    static constexpr int kCtas = PAIR ? 2 : 1;
    static constexpr int kRows = kCtaRows * kCtas, kCols = PAIR ? 256 : 64;
    static constexpr int kSide = kRows / kBox;                 // boxes of a block on the diagonal
    // A stage is kDepth boxes of the reduction: of each the left operand, and the CTA's part of the right one.
    static constexpr int kDepth = PAIR ? 1 : 2;
    static constexpr int kLeft = 2 * kBoxBytes, kRight = kCols / kCtas / kBox * kBoxBytes;
    static constexpr int kStageBytes = kDepth * (kLeft + kRight);
    static constexpr int kStages = PAIR ? 6 : 4;
    // half a box of staging for each group of 32 rows, two of them where there is more than one box
    static constexpr int kStaging = (kCols > kBox ? 2 : 1) * 4 * (kBoxBytes / 2);
    static constexpr int kSmem = kStages * kStageBytes + kStaging + 1024;   // and room to align them to 1024 bytes
    static constexpr int kTmemCols = 2 * kCols;
    // fp32 accumulator, fp16 operands; columns, and which way their rows lie, are added for each product
    static constexpr uint32_t kIdesc = 1u << 4 | uint32_t(kRows / 16) << 24;
};

struct OrthStep {
    float a, b, c, scale;    // scale: of B's operand
};
// Maps of a matrix of boxes, as [box row][box column][64][64]: copies of two boxes one above the other, of two
// side by side, of one.
struct BoxMaps {
    CUtensorMap down, beside, one;
};
struct OrthMaps {
    BoxMaps x[2], sa, sb;    // the operands
};
struct OrthParams {
    uint32_t* count;         // arrivals at the grid's barriers
    uint32_t* arrived;       // [A, A^2][tiles][CTAs of a tile]: splits of a product that are done
    float* d;                // [batch][mp]: diagonal of A
    float* e;                // [batch][mp]: diagonal of B
    uint8_t* x[2];           // operand of X, of even and odd steps
    uint8_t* xf;             // X in fp32, times x_scale
    uint8_t* af;             // A without its diagonal, in fp32
    uint8_t* sa;             // its operand
    uint8_t* sb;             // B without it
    float* part;             // splits' sums
    uint8_t* out;
    int64_t out_pitch, out_batch;   // bytes
    uint64_t limit_ns;
    float x_scale, a_scale;
    int32_t batch, m, n;     // of X as it is worked on (m <= n)
    int32_t bm, bn;          // boxes of m and n
    int32_t tiles;           // of A, of all matrices, at most
    int32_t cols[3];         // of a pair's tile
    int32_t steps, splits[3];  // of the reductions of A, A^2 and B X (the last always 1)
    int32_t turned;          // out is X^T
    int32_t wide;            // out takes 16-byte stores
    int32_t stall;
    OrthStep step[kMaxSteps];
};

// Boxes from column c and row r on into this CTA's shared memory; word of them goes to a barrier of the pair's first CTA.
template <bool PAIR>
__device__ __forceinline__ void bring(uint32_t dst, const CUtensorMap* map, int c, int r, uint32_t bar) {
    if constexpr (PAIR)
        asm volatile(
            "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %2, %3, %4}], [%5];" ::"r"(
                dst),
            "l"(map), "r"(0), "r"(c), "r"(r), "r"(bar)
            : "memory");
    else
        asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %3, %4}], [%5];" ::"r"(dst),
                     "l"(map), "r"(0), "r"(c), "r"(r), "r"(bar)
                     : "memory");
}
__device__ __forceinline__ uint32_t cluster_addr(uint32_t bar, int rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(bar), "r"(rank));
    return r;
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void cluster_meet() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Once the products issued so far are done: an arrival at the barrier (of both CTAs).
template <bool PAIR>
__device__ __forceinline__ void commit(uint32_t bar) {
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                     "h"(uint16_t(3))
                     : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(add)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
                     "l"(a), "l"(b), "r"(idesc), "r"(add)
                     : "memory");
}
// Descriptor of an operand: two boxes, 8 rows of 128 bytes 1024 bytes apart.  Rows
// along the reduction: the boxes hold 64 columns of the output each.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
    return uint64_t((addr & 0x3ffffu) >> 4) | uint64_t(kBoxBytes >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 |
           uint64_t(2) << 61;
}

__device__ __forceinline__ void tmem_ld8(uint32_t addr, float (&f)[8]) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(addr)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float (&f)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(r[i]);
}

// Sixteen columns from each of two places.
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float (&f)[16], uint32_t addr2, float (&g)[16]) {
    uint32_t r[16], q[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%33];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]),
          "=r"(q[4]), "=r"(q[5]), "=r"(q[6]), "=r"(q[7]), "=r"(q[8]), "=r"(q[9]), "=r"(q[10]), "=r"(q[11]), "=r"(q[12]), "=r"(q[13]),
          "=r"(q[14]), "=r"(q[15])
        : "r"(addr), "r"(addr2)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        f[i] = __uint_as_float(r[i]);
        g[i] = __uint_as_float(q[i]);
    }
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// 16-byte piece `p` (of 8) of row r in a box.
__device__ __forceinline__ uint32_t piece_at(int r, int p) { return uint32_t(r) * 128 + uint32_t((p ^ (r & 7)) * 16); }

template <bool PAIR>
__device__ __forceinline__ int cols_of(const OrthParams& p, int phase) { return PAIR ? p.cols[phase] : TileOf<PAIR>::kCols; }

// One piece of a product: a tile, or a split of its reduction.  i: the block of kRows rows, j: of the tile's columns, jb: the
// block on the diagonal that the columns are part of.
struct Item {
    int mat, i, j, jb, split, s0, stages, tile;
};
template <bool PAIR>
__device__ __forceinline__ Item item_of(const OrthParams& p, int phase, int at) {
    const int cols = cols_of<PAIR>(p, phase), in = TileOf<PAIR>::kRows / cols;   // tiles beside one another in such a block
    const int tm = p.bm / TileOf<PAIR>::kSide, tn = p.bn * kBox / cols;
    const int all = (phase == 0 ? p.bn : p.bm) / TileOf<PAIR>::kDepth, splits = p.splits[phase];
    Item w;
    const int t = at / splits;
    w.split = at - t * splits;
    const int per = (all + splits - 1) / splits;
    w.s0 = w.split * per;
    w.stages = min(per, all - w.s0);
    w.tile = t;
    if (phase == 2) {
        const int tiles = tm * tn;
        w.mat = t / tiles;
        const int k = t - w.mat * tiles;
        w.j = k / tm;
        w.i = k - w.j * tm;
        w.jb = 0;
    } else {
        const int tiles = tm * (tm + 1) / 2 * in;
        w.mat = t / tiles;
        const int k = (t - w.mat * tiles) / in;
        // block column j holds blocks [j (j + 1) / 2, ...)
        int j = int((sqrtf(8.0f * float(k) + 1.0f) - 1.0f) * 0.5f);
        while (j * (j + 1) / 2 > k) --j;
        while ((j + 1) * (j + 2) / 2 <= k) ++j;
        w.jb = j;
        w.i = k - j * (j + 1) / 2;
        w.j = j * in + t % in;
    }
    return w;
}
template <bool PAIR>
__device__ __forceinline__ int items_of(const OrthParams& p, int phase) {
    const int cols = cols_of<PAIR>(p, phase);
    const int tm = p.bm / TileOf<PAIR>::kSide, tn = p.bn * kBox / cols;
    return p.batch * (phase == 2 ? tm * tn : tm * (tm + 1) / 2 * (TileOf<PAIR>::kRows / cols)) * p.splits[phase];
}

// From which block of the reduction on an operand's boxes are read as its rows (before it, as its columns: a symmetric
// matrix has the boxes on and above the diagonal).
__device__ __forceinline__ int left_block(int phase, const Item& w) { return phase == 0 ? 0 : w.i; }
__device__ __forceinline__ int right_block(int phase, const Item& w) { return phase == 0 ? 0 : phase == 1 ? w.jb : 1 << 30; }

template <int N>
struct Step {
    static constexpr int value = N;
};
template <int N>
struct Ring {
    int at = 0;
    uint32_t round = 0;
    __device__ __forceinline__ void next() {
        if (++at == N) {
            at = 0;
            round ^= 1;
        }
    }
};

// Until `want` CTAs have arrived.
__device__ __forceinline__ bool grid_wait(const uint32_t* count, uint32_t want, uint64_t limit_ns) {
    uint64_t t0 = 0;
    for (uint64_t it = 1;; ++it) {
        uint32_t v;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(count) : "memory");
        if (v >= want) return true;
        if (it % 64) continue;
        const uint64_t t = global_ns();
        if (t0 == 0) t0 = t;
        else if (t - t0 > limit_ns || it > (uint64_t(1) << 40)) return false;
    }
}
// One lane of a warp.
__device__ __forceinline__ bool elected() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// mbar_wait_warp with a limit of its own.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, uint64_t limit_ns) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    uint64_t t0 = 0;
    for (uint64_t it = 1; it < (uint64_t(1) << 40); ++it) {
        if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
        if (it % kPollsPerTime) continue;
        const uint64_t t = __shfl_sync(0xffffffffu, global_ns(), 0);
        if (t0 == 0) t0 = t;
        else if (t - t0 > limit_ns) return false;
    }
    return false;
}
// A wait for the grid, in shared memory: as long as the grid may take.
__device__ __forceinline__ bool wait_long(uint32_t bar, uint32_t parity, uint64_t limit_ns) {
    uint64_t t0 = 0;
    for (uint64_t it = 1;; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if (it % kPollsPerTime) continue;
        const uint64_t t = global_ns();
        if (t0 == 0) t0 = t;
        else if (t - t0 > limit_ns || it > (uint64_t(1) << 40)) return false;
    }
}

// The warps that read the accumulators take one way: a wait that only some of them gave up on
// would leave the others at their barrier.
__device__ __forceinline__ bool sum_warps_agree(bool ok) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"(uint32_t(ok)), "n"(kSumWarps * 32)
        : "memory");
    return r != 0;
}

// The four warps with the same rows meet.
__device__ __forceinline__ void rows_meet(int quad) { asm volatile("bar.sync %0, 128;" ::"r"(2 + quad) : "memory"); }

__device__ __forceinline__ void sts128(uint32_t addr, const uint4& v) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t addr) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
    return v;
}

// 32 rows of 64 columns of the output, from 4 KB of staging in shared memory (rows of 128 bytes,
// swizzled), by four warps of which this is the `part`th.  r0, c0: the first row and column.
__device__ __forceinline__ void store_rows(const OrthParams& p, int mat, int r0, int c0, uint32_t stage, int part, int lane) {
    uint8_t* base = p.out + int64_t(mat) * p.out_batch;
    if (p.wide && c0 + kBox <= p.n) {
        const int piece = lane % 8;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int r = (k * 4 + part) * 4 + lane / 8;
            const uint4 v = lds128(stage + piece_at(r, piece));
            if (r0 + r < p.m) *reinterpret_cast<uint4*>(base + int64_t(r0 + r) * p.out_pitch + c0 * 2 + piece * 16) = v;
        }
        return;
    }
#pragma unroll 4
    for (int k = part; k < 64; k += 4) {
        const int r = k / 2, c = k % 2 * 32 + lane;
        const uint32_t v = lds16(stage + piece_at(r, c / 8) + c % 8 * 2);
        if (r0 + r < p.m && c0 + c < p.n) *reinterpret_cast<uint16_t*>(base + int64_t(r0 + r) * p.out_pitch + (c0 + c) * 2) = uint16_t(v);
    }
}
// A row's columns c .. c + 15 of an output that is X^T: the lanes' rows are neighbours there.
__device__ __forceinline__ void store_turned(const OrthParams& p, int mat, int r, int c, const float (&f)[kChunk]) {
    if (r >= p.m) return;
    uint8_t* o = p.out + int64_t(mat) * p.out_batch + int64_t(c) * p.out_pitch + int64_t(r) * 2;
#pragma unroll
    for (int k = 0; k < kChunk; ++k)
        if (c + k < p.n) *reinterpret_cast<__nv_bfloat16*>(o + k * p.out_pitch) = __float2bfloat16_rn(f[k]);
}

// Where fp32 matrices keep row r: rows in groups of 32, four columns of a group's rows after another, so that
// a warp with a row a lane reads and writes 512 bytes at once.
__device__ __forceinline__ int64_t row_at(int64_t mat, int rows, int cols, int r) {
    return ((mat * (rows / 32) + r / 32) * (cols / 4)) * 512 + r % 32 * 16;
}
__device__ __forceinline__ int quad_at(int c) { return c / 4 * 512; }

// A row of a product's tile on its way to the next operand, 8 or 16 columns at a time.
struct Finish {
    const OrthParams& p;
    const OrthStep& co;
    const int phase, gr;
    const bool final;
    const int mat;
    uint8_t* state;          // the row of A or of X in fp32
    uint8_t* out;            // the next operand: the row of boxes
    int64_t diag;            // of the matrix's first diagonal element
    float scale, cs, dr;
    float4 next[4], now[4];  // what is read beside the accumulator: A or X
    float d_next, d_now;     // A's diagonal, of a column a lane

    __device__ __forceinline__ Finish(const OrthParams& q, int ph, int step, bool fin, int m, int r)
        : p(q), co(q.step[step]), phase(ph), gr(r), final(fin), mat(m) {
        const int cols = (phase == 2 ? p.bn : p.bm) * kBox;
        state = (phase == 2 ? p.xf : p.af) + row_at(mat, p.bm * kBox, cols, gr);
        out = (phase == 0 ? p.sa : phase == 1 ? p.sb : p.x[step & 1 ^ 1]) + (int64_t(mat) * p.bm + gr / kBox) * (cols / kBox) * kBoxBytes;
        diag = int64_t(mat) * p.bm * kBox;
        cs = 0.0f;
        if (phase == 0) {
            scale = 1.0f / (p.x_scale * p.x_scale);
            dr = 0.0f;
        } else if (phase == 1) {
            scale = 1.0f / (p.a_scale * p.a_scale);
            cs = co.c * scale;
            dr = __ldcg(p.d + diag + gr);
        } else {
            scale = 1.0f / co.scale;
            dr = co.a + __ldcg(p.e + diag + gr);
        }
    }
    template <int N>
    __device__ __forceinline__ void ask(int col, int lane) {
        if (phase == 0) return;
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) next[k] = __ldcg(reinterpret_cast<const float4*>(state + quad_at(col + 4 * k)));
        if (phase == 1) d_next = __ldcg(p.d + diag + col + lane % (8 * N));
    }
    template <int N>
    __device__ __forceinline__ void take() {
#pragma unroll
        for (int k = 0; k < 2 * N; ++k) now[k] = next[k];
        d_now = d_next;
    }
    // Columns col .. col + 7 (all lanes): f from the accumulator, and what becomes of it as the next operand; k: which of the
    // eights asked for.
    __device__ __forceinline__ uint4 piece(int col, int k, float* f) {
        const float old[8] = {now[2 * k].x, now[2 * k].y, now[2 * k].z, now[2 * k].w, now[2 * k + 1].x, now[2 * k + 1].y, now[2 * k + 1].z, now[2 * k + 1].w};
        // the warp's rows meet these columns on the diagonal: seldom
        const bool diagonal = phase < 2 && (col & ~31) == (gr & ~31);
        float sc = 1.0f;
        if (phase == 0) {
#pragma unroll
            for (int m = 0; m < 8; ++m) f[m] *= scale;
            if (diagonal) {
                float on = 0.0f;
#pragma unroll
                for (int m = 0; m < 8; ++m) {
                    on = col + m == gr ? f[m] : on;
                    f[m] = col + m == gr ? 0.0f : f[m];
                }
                if (col <= gr && gr < col + 8) __stcg(p.d + diag + gr, on);
            }
            sc = p.a_scale;
        } else if (phase == 1) {
            // b A0 + c (A0^2 + (d_i + d_j) A0)
            float on = 0.0f;
            if (diagonal) {
#pragma unroll
                for (int m = 0; m < 8; ++m) on = col + m == gr ? f[m] : on;
            }
            const float bc = fmaf(co.c, dr, co.b);
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const float dj = __shfl_sync(0xffffffffu, d_now, 8 * k + m);
                f[m] = fmaf(fmaf(co.c, dj, bc), old[m], cs * f[m]);
            }
            if (diagonal) {
#pragma unroll
                for (int m = 0; m < 8; ++m) f[m] = col + m == gr ? 0.0f : f[m];
                // (A0 is zero there)
                if (col <= gr && gr < col + 8) __stcg(p.e + diag + gr, fmaf(cs, on, dr * bc));
            }
            sc = co.scale;
        } else {
#pragma unroll
            for (int m = 0; m < 8; ++m) f[m] = fmaf(dr, old[m], f[m] * scale);
        }
        if (phase == 0 || (phase == 2 && !final)) {
            __stcg(reinterpret_cast<float4*>(state + quad_at(col)), make_float4(f[0], f[1], f[2], f[3]));
            __stcg(reinterpret_cast<float4*>(state + quad_at(col + 4)), make_float4(f[4], f[5], f[6], f[7]));
        }
        return make_uint4(pack_f16(f[0] * sc, f[1] * sc), pack_f16(f[2] * sc, f[3] * sc), pack_f16(f[4] * sc, f[5] * sc),
                          pack_f16(f[6] * sc, f[7] * sc));
    }
};

template <bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) orth_product_kernel(const __grid_constant__ OrthMaps maps, const __grid_constant__ OrthParams p) {
    using Tile = TileOf<PAIR>;
    constexpr int kCtas = Tile::kCtas, kStages = Tile::kStages, kStageBytes = Tile::kStageBytes;
    constexpr int kCols = Tile::kCols, kTmemCols = Tile::kTmemCols, kSide = Tile::kSide;
    extern __shared__ uint8_t raw[];
    // full: both CTAs' copies of a stage have landed (the first CTA's).  empty: its products are done (each CTA's own).
    // summed: an accumulator is complete; taken: it has been read (the first CTA's).  go: the grid has come to the next
    // product.
    __shared__ __align__(8) uint64_t bars[2 * kStages + 5];
    __shared__ uint32_t tmem_base;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = PAIR ? int(blockIdx.x & 1) : 0, unit = int(blockIdx.x) / kCtas, units = int(gridDim.x) / kCtas;
    const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t full = smem_addr(bars), empty = full + 8 * kStages;
    const uint32_t summed = empty + 8 * kStages, taken = summed + 16, go = taken + 16;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(summed + 8 * i, 1);
            mbar_init(taken + 8 * i, kCtas * kSumWarps);
        }
        mbar_init(go, 1);
        mbar_init_fence();
    }
    if (warp == 1) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base)), "r"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base)), "r"(kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (PAIR) cluster_meet();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    const int phases = 3 * p.steps;

    // Both of the next warps go through their loops as one, and one lane issues: what the copies and the products
    // are given is then computed once for the warp, in its uniform registers.  (One lane by itself took 0.30 us for
    // 64 of the reduction on a single CTA's tile, whatever came with them; three stages in flight were as fast as eight.  So 0.21, and
    // 0.17 with 128 a stage.)
    if (warp == 0) {
        // --- the operands ---
        Ring<kStages> st;
        const bool one = elected();
        const uint32_t first_full = PAIR ? cluster_addr(full, 0) : full;
        int it = 0;
        bool ok = true;
        for (int ph = 0; ph < phases && ok; ++ph) {
            const int phase = ph % 3;
            if (ph) ok = __all_sync(0xffffffffu, lane != 0 || grid_wait(p.count, uint32_t(ph) * gridDim.x, p.limit_ns));
            if (!ok) break;
            if (one) {
                asm volatile("fence.proxy.async.global;" ::: "memory");   // what they wrote is read by copies
                mbar_arrive(go);
            }
            const BoxMaps &xm = maps.x[ph / 3 & 1], &sm = phase == 1 ? maps.sa : maps.sb;
            const int items = items_of<PAIR>(p, phase), boxes = cols_of<PAIR>(p, phase) / kCtas / kBox;   // of the right operand
            const uint32_t bytes = kCtas * Tile::kDepth * (Tile::kLeft + boxes * kBoxBytes);
            const BoxMaps &lm = phase == 0 ? xm : sm, &rm = phase == 1 ? sm : xm;
            const CUtensorMap *const r_down = boxes == 1 ? &rm.one : &rm.down, *const r_beside = boxes == 1 ? &rm.one : &rm.beside;
            for (int i = unit; i < items && ok; i += units) {
                const Item w = item_of<PAIR>(p, phase, i);
                // first box row or column of this CTA's part of either operand
                const int left = w.i * kSide + rank * 2, right = (w.j * kCtas + rank) * boxes, r0 = w.mat * p.bm;
                const int lb = left_block(phase, w), rb = right_block(phase, w);
                for (int s = 0; s < w.stages; ++s, ++it, st.next()) {
                    ok = it < kStages || mbar_wait_warp(empty + 8 * st.at, st.round ^ 1);
                    if (!ok) break;
                    const int k0 = (w.s0 + s) * Tile::kDepth, kt = k0 / kSide;
                    const uint32_t to = ring + st.at * kStageBytes, bar = first_full + 8 * st.at;
                    if (one) {
                        if (rank == 0) mbar_expect_tx(full + 8 * st.at, bytes + (it == 0 && p.stall ? 16 : 0));
#pragma unroll
                        for (int d = 0; d < Tile::kDepth; ++d) {
                            const int k = k0 + d;
                            const uint32_t lt = to + d * Tile::kLeft, rt = to + Tile::kDepth * Tile::kLeft + d * Tile::kRight;
                            if (lb <= kt) bring<PAIR>(lt, &lm.down, k, r0 + left, bar);
                            else bring<PAIR>(lt, &lm.beside, left, r0 + k, bar);
                            if (rb <= kt) bring<PAIR>(rt, r_down, k, r0 + right, bar);
                            else bring<PAIR>(rt, r_beside, right, r0 + k, bar);
                        }
                    }
                    __syncwarp();
                }
            }
        }
        // every copy lands, and every arrival that ends a stage's products, before the CTA's memory is given back
        // (word of the second CTA's goes to the first; they have landed when their products are done, or long after).  Limited
        // waits, for that alone.
        for (int i = it > kStages ? it - kStages : 0; i < it && rank == 0; ++i)
            mbar_wait_warp(full + 8 * (i % kStages), (i / kStages) & 1);
        bool ended = true;
        for (int i = it > kStages ? it - kStages : 0; i < it && ended; ++i)
            ended = mbar_wait_warp(empty + 8 * (i % kStages), (i / kStages) & 1);
    } else if (warp == 1 && rank == 0) {
        // --- the products ---
        Ring<kStages> st;
        Ring<2> acc;
        const bool one = elected();
        int chunk = 0;
        bool ok = true;
        for (int ph = 0; ph < phases && ok; ++ph) {
            const int phase = ph % 3;
            const int items = items_of<PAIR>(p, phase);
            const uint32_t format = Tile::kIdesc | uint32_t(cols_of<PAIR>(p, phase) / 8) << 17;
            for (int i = unit; i < items && ok; i += units) {
                const Item w = item_of<PAIR>(p, phase, i);
                const int lb = left_block(phase, w), rb = right_block(phase, w);
                if (chunk >= 2) ok = mbar_wait_warp(taken + 8 * acc.at, acc.round ^ 1);
                for (int s = 0; s < w.stages && ok; ++s, st.next()) {
                    // (a first stage comes once the grid has come here)
                    ok = wait_warp(full + 8 * st.at, st.round, s ? kWaitNs : p.limit_ns);
                    if (!ok) break;
                    const int kt = (w.s0 + s) * Tile::kDepth / kSide;
                    const bool ta = lb > kt, tb = rb > kt;
                    const uint32_t idesc = format | (ta ? 1u << 15 : 0u) | (tb ? 1u << 16 : 0u);
                    if (one) {
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t l = operand_desc(ring + st.at * kStageBytes), r = l + (Tile::kDepth * Tile::kLeft >> 4);
                        // rows along the reduction: 16 of them are 2048 bytes further; across it 16 columns are 32 bytes
                        auto issue = [&](auto la, auto lb) {
#pragma unroll
                            for (int d = 0; d < Tile::kDepth; ++d)
#pragma unroll
                                for (int k = 0; k < kBox / 16; ++k)
                                    mma<PAIR>(tmem + acc.at * kCols, l + (d * Tile::kLeft >> 4) + k * la.value, r + (d * Tile::kRight >> 4) + k * lb.value,
                                              idesc, d > 0 || k > 0 || s > 0);
                        };
                        constexpr Step<2> across;
                        constexpr Step<(2048 >> 4)> along;
                        if (ta) tb ? issue(along, along) : issue(along, across);
                        else tb ? issue(across, along) : issue(across, across);
                        commit<PAIR>(empty + 8 * st.at);
                    }
                    __syncwarp();
                }
                if (ok && one) commit<PAIR>(summed + 8 * acc.at);
                __syncwarp();
                acc.next();
                ++chunk;
            }
        }
    } else if (warp >= kSumWarp) {
        // --- what comes of an accumulator ---
        const int quad = warp & 3, group = (warp - kSumWarp) >> 2, t = threadIdx.x - kSumWarp * 32;
        const int row = quad * 32 + lane;                 // of this CTA's 128
        const uint32_t first_taken = PAIR ? cluster_addr(taken, 0) : taken;
        const uint32_t from = tmem + (uint32_t(quad * 32) << 16);
        const uint32_t staging = ring + kStages * kStageBytes + quad * (kBoxBytes / 2);
        constexpr bool kTwo = kCols > kBox;
        int turn = 0;
        Ring<2> acc;
        bool ok = true;
        for (int ph = 0; ph < phases; ++ph) {
            const int phase = ph % 3, step = ph / 3;
            const bool final = ph == phases - 1;
            ok = sum_warps_agree(wait_long(go, ph & 1, p.limit_ns));
            if (!ok) break;
            const int splits = p.splits[phase], items = items_of<PAIR>(p, phase);
            const int cols = cols_of<PAIR>(p, phase);
            for (int i = unit; i < items; i += units, acc.next()) {
                const Item w = item_of<PAIR>(p, phase, i);
                Finish fin(p, phase, step, final, w.mat, w.i * Tile::kRows + rank * kCtaRows + row);
                const int c0 = w.j * cols + group * kChunk;   // the four groups of warps share every box's columns
                if (splits == 1) {
                    // what is read beside the accumulator is on its way before that is complete, and then a chunk ahead
                    fin.ask<2>(c0, lane);
                    ok = sum_warps_agree(mbar_wait_warp(summed + 8 * acc.at, acc.round));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
                    for (int c = 0; c < cols; c += kBox) {
                        float f[kChunk];
                        tmem_ld16(from + acc.at * kCols + group * kChunk + c, f);
                        if (c + kBox == cols) {
                            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                            __syncwarp();
                            if (lane == 0) arrive_at(first_taken + 8 * acc.at);
                        }
                        fin.take<2>();
                        if (c + kBox < cols) fin.ask<2>(c0 + c + kBox, lane);
                        uint4 v[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) v[k] = fin.piece(c0 + c + 8 * k, k, f + 8 * k);
                        if (final) {
                            const float back = 1.0f / p.x_scale;
#pragma unroll
                            for (int k = 0; k < kChunk; ++k) f[k] *= back;
                            if (p.turned) {
                                store_turned(p, w.mat, fin.gr, c0 + c, f);
                                continue;
                            }
#pragma unroll
                            for (int k = 0; k < 2; ++k)
                                v[k] = make_uint4(pack_bf16(f[8 * k], f[8 * k + 1]), pack_bf16(f[8 * k + 2], f[8 * k + 3]),
                                                  pack_bf16(f[8 * k + 4], f[8 * k + 5]), pack_bf16(f[8 * k + 6], f[8 * k + 7]));
                        }
                        // 32 rows of a box are one piece of memory.  Two halves of staging take turns: the one before this has
                        // been read when its store's thread comes to this one's meeting.
                        const uint32_t stage = staging + (kTwo ? turn : 0) * 4 * (kBoxBytes / 2);
                        if constexpr (!kTwo) {
                            if (group == 0 && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                            rows_meet(quad);
                        }
#pragma unroll
                        for (int k = 0; k < 2; ++k) sts128(stage + piece_at(lane, group * 2 + k), v[k]);
                        if (!final) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        if (kTwo && group == 0 && lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                        rows_meet(quad);
                        const int col = w.j * cols + c;
                        if (final) {
                            store_rows(p, w.mat, fin.gr - lane, col, stage, group, lane);
                        } else if (group == 0 && lane == 0) {
                            bulk_s2g(fin.out + int64_t(col / kBox) * kBoxBytes + quad % 2 * (kBoxBytes / 2), stage, kBoxBytes / 2);
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                        turn ^= 1;
                    }
                    continue;
                }
                // every CTA with a split of the tile leaves its sums and takes a share of the columns of all of them,
                // added in the splits' order (the items are no more than the CTAs, so all splits are on their way)
                ok = sum_warps_agree(mbar_wait_warp(summed + 8 * acc.at, acc.round));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const int size = kCtaRows * cols;
                float* parts = p.part + (int64_t(w.tile) * kCtas + rank) * splits * size + row;
                float* mine = parts + int64_t(w.split) * size;
                const uint32_t sums = from + acc.at * kCols;
                // eight columns are a piece; pieces 4 s .. 4 s + 3 are split s's, and so on, one for each group of warps
#pragma unroll 1
                for (int k = group; k < cols / 8; k += 4) {
                    if (k / 4 % splits == w.split) continue;
                    float f[8];
                    tmem_ld8(sums + k * 8, f);
#pragma unroll
                    for (int m = 0; m < 8; ++m) __stcg(mine + (k * 8 + m) * kCtaRows, f[m]);
                }
                asm volatile("bar.sync 1, %0;" ::"n"(kSumWarps * 32) : "memory");
                uint32_t* arrived = p.arrived + ((phase * p.tiles + w.tile) * kCtas + rank);
                if (t == 0) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(arrived) : "memory");
                // (the counters only grow: this product's splits come on top of the earlier steps')
                bool came = true;
                if (lane == 0) came = grid_wait(arrived, uint32_t(splits) * uint32_t(step + 1), p.limit_ns);
                ok = sum_warps_agree(__all_sync(0xffffffffu, came));
                if (!ok) break;
#pragma unroll 1
                for (int k = w.split * 4 + group; k < cols / 8; k += splits * 4) {
                    const int col = w.j * cols + k * 8;
                    fin.ask<1>(col, lane);
                    float own[8], f[8] = {};
                    tmem_ld8(sums + k * 8, own);
                    const float* at = parts + k * 8 * kCtaRows;
                    // three splits' loads at a time
#pragma unroll 1
                    for (int s = 0; s < splits; s += 3, at += 3 * size) {
                        float g[3][8];
#pragma unroll
                        for (int h = 0; h < 3; ++h)
#pragma unroll
                            for (int m = 0; m < 8; ++m) g[h][m] = s + h < splits && s + h != w.split ? __ldcg(at + h * size + m * kCtaRows) : 0.0f;
#pragma unroll
                        for (int h = 0; h < 3; ++h)
#pragma unroll
                            for (int m = 0; m < 8; ++m) f[m] += s + h == w.split ? own[m] : g[h][m];
                    }
                    fin.take<1>();
                    const uint4 v = fin.piece(col, 0, f);
                    *reinterpret_cast<uint4*>(fin.out + int64_t(col / kBox) * kBoxBytes + piece_at(fin.gr % kBox, col % kBox / 8)) = v;
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) arrive_at(first_taken + 8 * acc.at);
            }
            if (!ok) break;
            if (!final) {
                if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
                if (splits > 1) asm volatile("fence.proxy.async.global;" ::: "memory");   // (those store operands themselves)
                asm volatile("bar.sync 1, %0;" ::"n"(kSumWarps * 32) : "memory");
                if (t == 0) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p.count) : "memory");
            }
        }
        if (!ok) {
            // what is on its way out of shared memory ends first
            if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            // NaN where this CTA's outputs would be
            const int items = items_of<PAIR>(p, 2);
            for (int i = unit; i < items; i += units) {
                const Item w = item_of<PAIR>(p, 2, i);
                const int cols = cols_of<PAIR>(p, 2), r = w.i * Tile::kRows + rank * kCtaRows + row, c0 = w.j * cols + group * (cols / 4);
                for (int c = c0; c < min(c0 + cols / 4, p.n) && r < p.m; ++c)
                    *reinterpret_cast<uint16_t*>(p.out + int64_t(w.mat) * p.out_batch + int64_t(p.turned ? c : r) * p.out_pitch +
                                                 int64_t(p.turned ? r : c) * 2) = 0x7fff;
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncwarp();
    __syncthreads();
    if constexpr (PAIR) cluster_meet();   // the other CTA's barriers and operands are used until here
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

// --- before the products -----------------------------------------------------------

struct PrepParams {
    const uint8_t* u;
    uint8_t* m;              // momentum (null: none)
    float4* part;            // [batch][parts]: Squares
    uint32_t* zero;          // counters of the product kernel
    uint8_t* hi;
    uint8_t* xf;
    int64_t u_pitch, u_batch, m_pitch, m_batch;   // bytes
    int64_t rows, cols;      // as given; one long row where they are contiguous
    int32_t nzero, parts;
    float beta, x_scale;
    double eps;
    int32_t u_bf16, nesterov, turned, bm, bn;
    int32_t wide;            // rows on 16-byte boundaries
};

// Values c .. c + 7 of a row, zero beyond its end.
__device__ __forceinline__ void load8(const uint8_t* row, bool bf16, bool wide, int64_t c, int64_t cols, float (&f)[8]) {
    if (wide && c + 8 <= cols) {
        if (bf16) {
            unpack(*reinterpret_cast<const uint4*>(row + c * 2), f);
        } else {
            const float4 a = *reinterpret_cast<const float4*>(row + c * 4), b = *reinterpret_cast<const float4*>(row + c * 4 + 16);
            f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        f[k] = c + k >= cols ? 0.0f : bf16 ? to_f32(reinterpret_cast<const __nv_bfloat16*>(row)[c + k]) : reinterpret_cast<const float*>(row)[c + k];
}
// The momentum after a gradient, and the update that comes of both.
__device__ __forceinline__ float moved(const PrepParams& p, float m, float g) { return fmaf(1.0f - p.beta, g - m, m); }
__device__ __forceinline__ float update_of(const PrepParams& p, float m, float g) { return p.nesterov ? fmaf(p.beta, m - g, g) : m; }

// Sums of an update's squares: as they are, and of values times 2^-80 and 2^100 for a matrix whose squares leave fp32's
// range on either side.  A sum of plain squares from 2^-80 on has lost nothing that counts: what a square below 2^-126 loses is
// at most 2^-150, and 2^32 of them 2^-118.  Below it no value is above 2^-40, so the scaled squares stay below 2^120, and
// the smallest value of all, 2^-149, has one of 2^-98.  The scaled sums are added to where a thread's plain one
// says that they may be needed: below 2^-80, as all threads' are where the matrix's is, or above 2^60 (what it left out
// until then is nothing beside a sum beyond 2^128).
struct Squares {
    float plain = 0.0f, down = 0.0f, up = 0.0f;
    template <int N>
    __device__ __forceinline__ void count(const float (&f)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k) plain = fmaf(f[k], f[k], plain);
        if (plain < 0x1p-80f) {
#pragma unroll
            for (int k = 0; k < N; ++k) up = fmaf(f[k] * 0x1p100f, f[k] * 0x1p100f, up);
        } else if (plain > 0x1p60f) {
#pragma unroll
            for (int k = 0; k < N; ++k) down = fmaf(f[k] * 0x1p-80f, f[k] * 0x1p-80f, down);
        }
    }
    __device__ __forceinline__ void add(const float4& v) {
        plain += v.x;
        down += v.y;
        up += v.z;
    }
    __device__ __forceinline__ float4 all() const { return make_float4(plain, down, up, 0.0f); }
    // over a warp's lanes
    __device__ __forceinline__ void join() {
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            plain += __shfl_xor_sync(0xffffffffu, plain, o);
            down += __shfl_xor_sync(0xffffffffu, down, o);
            up += __shfl_xor_sync(0xffffffffu, up, o);
        }
    }
    // What an update is multiplied by, one factor after the other, to be X times x_scale: a power of two that brings very
    // large and very small values near 1, and the rest.
    __device__ __forceinline__ void factors(float x_scale, double eps, float (&f)[2]) const {
        const bool large = plain > 3.402823466e38f;
        const double norm = large ? sqrt(double(down)) * 0x1p80 : plain < 0x1p-80f ? sqrt(double(up)) * 0x1p-100 : sqrt(double(plain));
        const double to = double(x_scale) / (norm + eps);
        f[0] = large ? 0x1p-64f : 1.0f;
        f[1] = float(to * (large ? 0x1p64 : 1.0));
        if (to > 0x1p100) {
            // (zeros over an eps of next to nothing are zeros, over none NaN)
            f[0] = 0x1p100f;
            f[1] = norm + eps > 0.0 ? float(fmin(to * 0x1p-100, 3.4e38)) : __uint_as_float(0x7f800000u);
        }
    }
};

// Moves the momentum and leaves sums of the update's squares, one set a CTA.
__global__ void __launch_bounds__(256) orth_norm_kernel(PrepParams p) {
    __shared__ float4 sums[8];
    const int mat = blockIdx.y;
    if (mat == 0)
        for (int i = int(blockIdx.x) * 256 + int(threadIdx.x); i < p.nzero; i += p.parts * 256) p.zero[i] = 0;
    const uint8_t* u = p.u + int64_t(mat) * p.u_batch;
    uint8_t* m = p.m ? p.m + int64_t(mat) * p.m_batch : nullptr;
    const int64_t width = (p.cols + 7) / 8, all = p.rows * width, step = int64_t(p.parts) * 256;
    Squares s;
    // two eights at a time, all of them asked for before the first is worked on
    for (int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x; at < all; at += 2 * step) {
        float f[2][8], v[2][8];
        int64_t r[2], c[2];
        const bool two = at + step < all;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            split_item(h && two ? at + step : at, width, r[h], c[h]);
            c[h] *= 8;
            load8(u + r[h] * p.u_pitch, p.u_bf16, p.wide, c[h], p.cols, f[h]);
        }
        if (m) {
#pragma unroll
            for (int h = 0; h < 2; ++h) load8(m + r[h] * p.m_pitch, false, p.wide, c[h], p.cols, v[h]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (h && !two) break;
            if (m) {
                float* row = reinterpret_cast<float*>(m + r[h] * p.m_pitch) + c[h];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[h][k] = moved(p, v[h][k], f[h][k]);
                    f[h][k] = update_of(p, v[h][k], f[h][k]);
                }
                if (p.wide && c[h] + 8 <= p.cols) {
                    *reinterpret_cast<float4*>(row) = make_float4(v[h][0], v[h][1], v[h][2], v[h][3]);
                    *reinterpret_cast<float4*>(row + 4) = make_float4(v[h][4], v[h][5], v[h][6], v[h][7]);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (c[h] + k < p.cols) row[k] = v[h][k];
                }
            }
            s.count(f[h]);
        }
    }
    s.join();
    if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = s.all();
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < 8; ++w) s.add(sums[w]);
    p.part[int64_t(mat) * p.parts + blockIdx.x] = s.all();
}

// The update over its norm as X: operand and fp32, box by box.
__global__ void __launch_bounds__(256, 6) orth_split_kernel(PrepParams p) {
    __shared__ float4 sums[8];
    __shared__ float factor[2];
    __shared__ float tile[kBox][kBox + 1];
    const int mat = blockIdx.y, t = threadIdx.x;
    Squares s;
    for (int i = t; i < p.parts; i += 256) s.add(p.part[int64_t(mat) * p.parts + i]);
    s.join();
    if (t % 32 == 0) sums[t / 32] = s.all();
    __syncthreads();
    if (t == 0) {
        for (int w = 1; w < 8; ++w) s.add(sums[w]);
        s.factors(p.x_scale, p.eps, factor);
    }
    __syncthreads();
    const float f0 = factor[0], f1 = factor[1];
    const uint8_t* u = p.u + int64_t(mat) * p.u_batch;
    const uint8_t* m = p.m ? p.m + int64_t(mat) * p.m_batch : nullptr;
    const int r = t / 4, c = t % 4 * 16;     // a thread's row and its 16 columns of it
    const int64_t boxes = int64_t(p.bm) * p.bn;
    for (int64_t box = blockIdx.x; box < boxes; box += gridDim.x) {
        const int64_t br = box / p.bn, bc = box - br * p.bn;
        // the box of U: where X is turned, (bc, br)
        const int64_t ur = (p.turned ? bc : br) * kBox + r, uc = (p.turned ? br : bc) * kBox + c;
        float f[16];
        if (ur < p.rows && uc < p.cols) {
            float h[8];
#pragma unroll
            for (int k = 0; k < 16; k += 8) {
                load8(u + ur * p.u_pitch, p.u_bf16, p.wide, uc + k, p.cols, h);
                if (m) {
                    float v[8];
                    load8(m + ur * p.m_pitch, false, p.wide, uc + k, p.cols, v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[j] = update_of(p, v[j], h[j]);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) f[k + j] = uc + k + j < p.cols ? h[j] * f0 * f1 : 0.0f;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 16; ++k) f[k] = 0.0f;
        }
        if (p.turned) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 16; ++k) tile[r][c + k] = f[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 16; ++k) f[k] = tile[c + k][r];
        }
        const int64_t off = (int64_t(mat) * boxes + box) * kBoxBytes;
        uint8_t* const xf = p.xf + row_at(mat, p.bm * kBox, p.bn * kBox, int(br) * kBox + r) + quad_at(int(bc) * kBox + c);
#pragma unroll
        for (int k = 0; k < 16; k += 4) *reinterpret_cast<float4*>(xf + quad_at(k)) = make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]);
#pragma unroll
        for (int k = 0; k < 16; k += 8)
            *reinterpret_cast<uint4*>(p.hi + off + piece_at(r, (c + k) / 8)) =
                make_uint4(pack_f16(f[k], f[k + 1]), pack_f16(f[k + 2], f[k + 3]), pack_f16(f[k + 4], f[k + 5]), pack_f16(f[k + 6], f[k + 7]));
    }
}

// --- small matrices --------------------------------------------------------------------

// Up to 128 rows: a cluster has a matrix, each CTA up to 256 of its columns for the whole call, from the
// update to the output.  X lies in tensor memory in fp32 and in shared memory as operand.  A step needs the
// other CTAs once: their parts of A are added up, each CTA a share of the rows, through the cluster's shared
// memory, and A goes to all; A^2 is computed by each (128 x 128 x 128 takes less than sending it).
constexpr int kSmallRows = 128, kSmallCols = 256, kSmallThreads = 512, kSmallCtas = 16;
constexpr int kQuadPitch = kSmallRows * 16 + 16;   // of fp32 staging: four columns of all rows; 16 more keep eight quads of a row in eight banks
// X's operand, A's, and the other CTAs' sums; staging lies over them
constexpr int kSmallX = kSmallRows * kSmallCols * 2, kSmallA = kSmallRows * kSmallRows * 2;
constexpr int kSmallSums = kSmallRows * kSmallRows * 4 + kSmallCtas * 32 * 16;
constexpr int kSmallSmem = kSmallX + kSmallA + kSmallSums + 1024;
static_assert(kSmallCols / 4 * kQuadPitch <= kSmallX + kSmallA + kSmallSums, "staging");

struct SmallParams {
    const uint8_t* u;
    uint8_t* m;
    uint8_t* out;
    int64_t u_pitch, u_batch, m_pitch, m_batch, out_pitch, out_batch;   // bytes
    int64_t rows, cols;      // as given
    double eps;
    float beta, x_scale, a_scale;
    int32_t ctas, u_bf16, nesterov, turned, steps;
    int32_t stall;           // test switch: nobody hears of the first product
    int32_t wide, out_wide;  // rows on 16-byte boundaries
    OrthStep step[kMaxSteps];
};

__device__ __forceinline__ void tmem_st16(uint32_t addr, const float (&f)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n\t"
        "tcgen05.wait::st.sync.aligned;" ::"r"(addr),
        "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]), "f"(f[8]), "f"(f[9]), "f"(f[10]), "f"(f[11]),
        "f"(f[12]), "f"(f[13]), "f"(f[14]), "f"(f[15])
        : "memory");
}
__device__ __forceinline__ float4 lds_quad(uint32_t addr) {
    const uint4 v = lds128(addr);
    return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
}
// Stores into a CTA of the cluster.
__device__ __forceinline__ void st_cluster(uint32_t addr, const float4& v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, const uint4& v) {
    asm volatile("st.shared::cluster.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

// Where an operand of 128 rows keeps row r's columns c .. c + 7: boxes of 64 columns, two of rows each.
__device__ __forceinline__ uint32_t small_at(int r, int c) { return (c / kBox * 2 + r / kBox) * kBoxBytes + piece_at(r % kBox, c % kBox / 8); }
// Descriptor of an operand whose rows run along the reduction; the next 64 columns are two boxes further.
__device__ __forceinline__ uint64_t small_desc(uint32_t addr) {
    return uint64_t((addr & 0x3ffffu) >> 4) | uint64_t(2 * kBoxBytes >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}

__device__ __forceinline__ float element(const uint8_t* row, bool bf16, int64_t c) {
    return bf16 ? to_f32(reinterpret_cast<const __nv_bfloat16*>(row)[c]) : reinterpret_cast<const float*>(row)[c];
}
// Values c .. c + 3 of a row, zero beyond its end.
__device__ __forceinline__ float4 load_quad(const uint8_t* row, bool bf16, bool wide, int64_t c, int64_t cols) {
    if (wide && c + 4 <= cols) {
        if (!bf16) return *reinterpret_cast<const float4*>(row + c * 4);
        const uint2 v = *reinterpret_cast<const uint2*>(row + c * 2);
        return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                           __uint_as_float(v.y & 0xffff0000u));
    }
    return make_float4(c < cols ? element(row, bf16, c) : 0.0f, c + 1 < cols ? element(row, bf16, c + 1) : 0.0f,
                       c + 2 < cols ? element(row, bf16, c + 2) : 0.0f, c + 3 < cols ? element(row, bf16, c + 3) : 0.0f);
}

__device__ __forceinline__ void sts_quad(uint32_t addr, const float4& v) {
    sts128(addr, make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)));
}
// Four by four values and their transpose.
__device__ __forceinline__ void turn(float4 (&v)[4]) {
    const float4 a = v[0], b = v[1], c = v[2], d = v[3];
    v[0] = make_float4(a.x, b.x, c.x, d.x);
    v[1] = make_float4(a.y, b.y, c.y, d.y);
    v[2] = make_float4(a.z, b.z, c.z, d.z);
    v[3] = make_float4(a.w, b.w, c.w, d.w);
}
// Four values of an output's row of `cols` from c.
__device__ __forceinline__ void store_quad(uint8_t* row, bool wide, int64_t c, int64_t cols, const float4& v) {
    __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(row) + c;
    if (wide && c + 4 <= cols) {
        *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
        return;
    }
    if (c < cols) o[0] = __float2bfloat16_rn(v.x);
    if (c + 1 < cols) o[1] = __float2bfloat16_rn(v.y);
    if (c + 2 < cols) o[2] = __float2bfloat16_rn(v.z);
    if (c + 3 < cols) o[3] = __float2bfloat16_rn(v.w);
}

// K: a CTA's columns over 64.
template <int K>
__global__ void __launch_bounds__(kSmallThreads, 1) orth_small_kernel(const __grid_constant__ SmallParams p) {
    constexpr int kN = 64 * K, kMine = kN / 4;   // columns of the CTA, of a thread
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t done_bar;
    __shared__ uint32_t tmem_base;
    __shared__ __align__(16) float d[kSmallRows], e[kSmallRows];
    __shared__ __align__(16) float4 sums[kSmallThreads / 32], all[kSmallCtas];
    __shared__ float factor[2];
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, quad = warp & 3, group = warp >> 2, row = quad * 32 + lane;
    const int C = p.ctas, rank = int(blockIdx.x) % C, mat = int(blockIdx.x) / C;
    const uint32_t xs = (smem_addr(raw) + 1023) & ~1023u, as = xs + kSmallX, ss = as + kSmallA, done = smem_addr(&done_bar);
    if (t == 0) {
        mbar_init(done, 1);
        mbar_init_fence();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    // (the others' shared memory is written once they have started)
    __syncwarp();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    // --- the update, and its norm ---
    const uint8_t* u = p.u + int64_t(mat) * p.u_batch;
    uint8_t* m = p.m ? p.m + int64_t(mat) * p.m_batch : nullptr;
    const int64_t first = int64_t(rank) * kN;    // X's first column here
    const int64_t n = p.turned ? p.rows : p.cols;
    const int rows = int(p.turned ? p.cols : p.rows);
    Squares s;
    auto count = [&](const float4& v) {
        const float f[4] = {v.x, v.y, v.z, v.w};
        s.count(f);
    };
    // values c .. c + 3 of a row of `cols` move its momentum and become what comes of it
    auto move = [&](float* at, int64_t c, int64_t cols, float4& v) {
        float4 w = load_quad(reinterpret_cast<const uint8_t*>(at), false, p.wide, c, cols);
        auto one = [&](float& x, float& mom) {
            mom = fmaf(1.0f - p.beta, x - mom, mom);
            x = p.nesterov ? fmaf(p.beta, mom - x, x) : mom;
        };
        one(v.x, w.x);
        one(v.y, w.y);
        one(v.z, w.z);
        one(v.w, w.w);
        at += c;
        if (p.wide && c + 4 <= cols) {
            *reinterpret_cast<float4*>(at) = w;
        } else {
            at[0] = w.x;
            if (c + 1 < cols) at[1] = w.y;
            if (c + 2 < cols) at[2] = w.z;
            if (c + 3 < cols) at[3] = w.w;
        }
    };
    // through shared memory to a row a lane
    if (p.turned) {
        // a row of the update is a column of X: a lane has four neighbours of four of them
        for (int q = warp; q < kN / 4; q += kSmallThreads / 32) {
            const int r = lane * 4;
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t c = first + q * 4 + k;
                v[k] = c < n ? load_quad(u + c * p.u_pitch, p.u_bf16, p.wide, r, rows) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
            if (m) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (first + q * 4 + k < n && r < rows) move(reinterpret_cast<float*>(m + (first + q * 4 + k) * p.m_pitch), r, rows, v[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) count(v[k]);
            turn(v);
#pragma unroll
            for (int k = 0; k < 4; ++k) sts_quad(xs + q * kQuadPitch + (r + k) * 16, v[k]);
        }
    } else {
        // eight lanes a row, four rows a warp
#pragma unroll 4
        for (int i = warp; i < kN / 32 * (kSmallRows / 4); i += kSmallThreads / 32) {
            const int q = i % (kN / 32) * 8 + lane % 8, r = i / (kN / 32) * 4 + lane / 8;
            const int64_t c = first + q * 4;
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (r < rows && c < n) {
                v = load_quad(u + r * p.u_pitch, p.u_bf16, p.wide, c, n);
                if (m) move(reinterpret_cast<float*>(m + r * p.m_pitch), c, n, v);
                count(v);
            }
            sts_quad(xs + q * kQuadPitch + r * 16, v);
        }
    }
    s.join();
    if (lane == 0) sums[warp] = s.all();
    __syncthreads();
    float x[kMine];
#pragma unroll
    for (int k = 0; k < kMine; k += 4) {
        const float4 v = lds_quad(xs + (group * kMine + k) / 4 * kQuadPitch + row * 16);
        x[k] = v.x;
        x[k + 1] = v.y;
        x[k + 2] = v.z;
        x[k + 3] = v.w;
    }
    __syncwarp();
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (t < C) {
        s = Squares();
        for (int w = 0; w < kSmallThreads / 32; ++w) s.add(sums[w]);
        st_cluster(cluster_addr(smem_addr(&all[rank]), t), s.all());
    }
    cluster_meet();
    if (t == 0) {
        s = Squares();
        for (int k = 0; k < C; ++k) s.add(all[k]);
        s.factors(p.x_scale, p.eps, factor);
    }
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base, mine = uint32_t(quad * 32) << 16;
    const uint32_t state = tmem + mine + kSmallCols + group * kMine;
    const bool real = row < rows;
    {
        const float f0 = factor[0], f1 = factor[1];
#pragma unroll
        for (int c = 0; c < kMine; c += 16) {
            float f[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) f[k] = real && first + group * kMine + c + k < n ? x[c + k] * f0 * f1 : 0.0f;
            tmem_st16(state + c, f);
#pragma unroll
            for (int k = 0; k < 16; k += 8)
                sts128(xs + small_at(row, group * kMine + c + k), make_uint4(pack_f16(f[k], f[k + 1]), pack_f16(f[k + 2], f[k + 3]),
                                                                            pack_f16(f[k + 4], f[k + 5]), pack_f16(f[k + 6], f[k + 7])));
        }
    }
    // --- the steps ---
    uint8_t* const out = p.out + int64_t(mat) * p.out_batch;
    const float x_back = 1.0f / p.x_scale;
    uint32_t round = 0;
    bool ok = true;
    // everybody's writes are in place, one thread issues the products, and everybody waits for them.  After a wait of its own
    // that ran out it issues no more (the others' next wait runs out too), so that one product at most is unaccounted for.
    auto products = [&](auto issue) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncthreads();
        if (warp == 0) {
            if (lane == 0 && ok) {
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                issue();
                if (!p.stall) commit<false>(done);
            }
            __syncwarp();
        }
        ok = ok && mbar_wait_bounded(done, round, kWaitNs);
        if (ok) round ^= 1;
        __syncwarp();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    };
    constexpr uint32_t kFormat = 1u << 4 | uint32_t(kSmallRows / 16) << 24;
    constexpr uint32_t kSquare = kFormat | uint32_t(kSmallRows / 8) << 17, kOnX = kFormat | uint32_t(kN / 8) << 17 | 1u << 16;
    const uint32_t from = tmem + mine + group * 32;
    for (int step = 0; step < p.steps; ++step) {
        const OrthStep co = p.step[step];
        // A, of this CTA's columns
        products([&]() {
#pragma unroll
            for (int j = 0; j < K; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint64_t o = operand_desc(xs + j * 2 * kBoxBytes) + 2 * k;
                    mma<false>(tmem, o, o, kSquare, j > 0 || k > 0);
                }
        });
        // A as its operand, times a_scale; the diagonal (in the warps whose columns are their rows) by itself
        const bool diagonal = group == quad;
        const float to_a = p.a_scale / (p.x_scale * p.x_scale), nan = __uint_as_float(0x7fffffffu);
        float f[32];
        {
            float g[16], h[16];
            tmem_ld16(from, g, from + 16, h);
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                f[k] = g[k];
                f[16 + k] = h[k];
            }
        }
        if (!ok) {
#pragma unroll
            for (int k = 0; k < 32; ++k) f[k] = nan;
        }
        if (C == 1) {
            if (diagonal) {
                float on = 0.0f;
#pragma unroll
                for (int k = 0; k < 32; ++k) {
                    on = k == lane ? f[k] : on;
                    f[k] = k == lane ? 0.0f : f[k];
                }
                d[row] = on * to_a;
            }
#pragma unroll
            for (int k = 0; k < 32; k += 8) {
                uint32_t w[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const float2 v = mul2(make_float2(f[k + 2 * h], f[k + 2 * h + 1]), both(to_a));
                    w[h] = pack_f16(v.x, v.y);
                }
                sts128(as + small_at(row, group * 32 + k), make_uint4(w[0], w[1], w[2], w[3]));
            }
        } else {
            // (plain stores and the cluster's barrier: stores that a barrier of the receiver counts, without waiting for all,
            // took 46 us a call for 43 with two CTAs, 54 for 57 with sixteen)
            // a CTA adds up 128 / C rows, in the CTAs' order; four columns of these rows are one piece (and 16 bytes more,
            // so that pieces of a row lie in different banks)
            const int each = kSmallRows / C, pitch = each * 16 + 16;
            const uint32_t to = cluster_addr(ss + rank * 32 * pitch + row % each * 16, row / each);
#pragma unroll
            for (int k = 0; k < 8; ++k) st_cluster(to + (group * 8 + k) * pitch, make_float4(f[4 * k], f[4 * k + 1], f[4 * k + 2], f[4 * k + 3]));
            cluster_meet();
            for (int i = t; i < each * 16; i += kSmallThreads) {
                // eight columns of a row, eight neighbours of which a lane group sends on as 128 bytes
                const int r = i / 16, c = i % 16 * 8, full = rank * each + r;
                float v[8] = {};
                for (int k = 0; k < C; ++k) {
                    const uint32_t at = ss + (k * 32 + c / 4) * pitch + r * 16;
                    const float4 a = lds_quad(at), b = lds_quad(at + pitch);
                    v[0] += a.x, v[1] += a.y, v[2] += a.z, v[3] += a.w;
                    v[4] += b.x, v[5] += b.y, v[6] += b.z, v[7] += b.w;
                }
                float on = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    v[k] *= to_a;
                    on = c + k == full ? v[k] : on;
                    v[k] = c + k == full ? 0.0f : v[k];
                }
                const uint4 w = make_uint4(pack_f16(v[0], v[1]), pack_f16(v[2], v[3]), pack_f16(v[4], v[5]), pack_f16(v[6], v[7]));
                const uint32_t at = as + small_at(full, c), d_at = smem_addr(&d[full]);
                for (int k = 0; k < C; ++k) {
                    st_cluster(cluster_addr(at, k), w);
                    if (c / 8 == full / 8) st_cluster(cluster_addr(d_at, k), on);
                }
            }
            asm volatile("fence.proxy.async;" ::: "memory");
            cluster_meet();
        }
        // A0^2, and B in A's place
        products([&]() {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint64_t o = operand_desc(as + k / 4 * 2 * kBoxBytes) + 2 * (k % 4);
                mma<false>(tmem, o, o, kSquare, k > 0);
            }
        });
        {
            // b A0 + c (A0^2 + (d_i + d_j) A0), times B's scale; here A0, d and A0^2 are times a_scale (A0^2 twice)
            const float back = 1.0f / p.a_scale, dr = d[row], to_b = co.c * back * back * co.scale;
            const float2 cs = both(to_b), bc = both(fmaf(to_b, dr, co.b * back * co.scale));
            float g2[2][16];
            tmem_ld16(from, g2[0], from + 16, g2[1]);
#pragma unroll
            for (int c = 0; c < 32; c += 16) {
                float(&g)[16] = g2[c / 16];
                if (diagonal) {
                    // (A0 is zero there)
                    float on = 0.0f;
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        on = c + k == lane ? g[k] : on;
                        g[k] = c + k == lane ? 0.0f : g[k];
                    }
                    const float dt = dr * back;
                    if (lane / 16 == c / 16) e[row] = fmaf(co.c * back * back, on, dt * fmaf(co.c, dt, co.b));
                }
#pragma unroll
                for (int k = 0; k < 16; k += 8) {
                    const int col = group * 32 + c + k;
                    const uint32_t at = as + small_at(row, col);
                    const uint4 a = lds128(at);
                    const uint32_t aw[4] = {a.x, a.y, a.z, a.w};
                    const float4 d0 = *reinterpret_cast<const float4*>(d + col), d1 = *reinterpret_cast<const float4*>(d + col + 4);
                    const float2 dj[4] = {make_float2(d0.x, d0.y), make_float2(d0.z, d0.w), make_float2(d1.x, d1.y), make_float2(d1.z, d1.w)};
                    uint32_t w[4];
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const float2 a2 = __half22float2(*reinterpret_cast<const __half2*>(&aw[h]));
                        const float2 v = fma2(fma2(cs, dj[h], bc), a2, mul2(cs, make_float2(g[k + 2 * h], g[k + 2 * h + 1])));
                        w[h] = pack_f16(v.x, v.y);
                    }
                    sts128(at, make_uint4(w[0], w[1], w[2], w[3]));
                }
            }
        }
        // X
        products([&]() {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                mma<false>(tmem, operand_desc(as + k / 4 * 2 * kBoxBytes) + 2 * (k % 4),
                           small_desc(xs + k / 4 * kBoxBytes) + (2048 >> 4) * (k % 4), kOnX, k > 0);
        });
        const float back = 1.0f / co.scale, keep = co.a + e[row];
#pragma unroll
        for (int c = 0; c < kMine; c += 16) {
            float g[16], h[16];
            tmem_ld16(tmem + mine + group * kMine + c, g, state + c, h);
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
                const float2 v = fma2(both(keep), make_float2(h[k], h[k + 1]), mul2(make_float2(g[k], g[k + 1]), both(back)));
                g[k] = v.x;
                g[k + 1] = v.y;
            }
            if (step < p.steps - 1) {
                tmem_st16(state + c, g);
#pragma unroll
                for (int k = 0; k < 16; k += 8)
                    sts128(xs + small_at(row, group * kMine + c + k), make_uint4(pack_f16(g[k], g[k + 1]), pack_f16(g[k + 2], g[k + 3]),
                                                                                pack_f16(g[k + 4], g[k + 5]), pack_f16(g[k + 6], g[k + 7])));
                continue;
            }
            // --- the output ---
#pragma unroll
            for (int k = 0; k < 16; ++k) g[k] = ok ? g[k] * x_back : __uint_as_float(0x7fffffffu);
            // the operands have been read: their place is staging again
#pragma unroll
            for (int k = 0; k < 16; k += 4)
                sts_quad(xs + (group * kMine + c + k) / 4 * kQuadPitch + row * 16, make_float4(g[k], g[k + 1], g[k + 2], g[k + 3]));
        }
    }
    __syncthreads();
    if (p.turned) {
        for (int q = warp; q < kN / 4; q += kSmallThreads / 32) {
            const int r = lane * 4;
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = lds_quad(xs + q * kQuadPitch + (r + k) * 16);
            turn(v);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (first + q * 4 + k < n) store_quad(out + (first + q * 4 + k) * p.out_pitch, p.out_wide, r, rows, v[k]);
        }
    } else {
        for (int i = warp; i < kN / 32 * (kSmallRows / 4); i += kSmallThreads / 32) {
            const int q = i % (kN / 32) * 8 + lane % 8, r = i / (kN / 32) * 4 + lane / 8;
            if (r < rows) store_quad(out + r * p.out_pitch, p.out_wide, first + q * 4, n, lds_quad(xs + q * kQuadPitch + r * 16));
        }
    }
    // (the product that was given up on uses the CTA's memory until it is done)
    if (!ok && t == 0) mbar_wait_bounded(done, round, kDrainNs);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// --- host -------------------------------------------------------------------------

constexpr int64_t al(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// How a call is cut, and where its parts lie in the workspace.
struct Plan {
    int64_t batch, m, n, bm, bn, tm;
    bool pair, turned;
    int ctas;                 // of a tile
    int64_t cols[3], splits[3], tiles[3], items[3], half, parts;   // half: tiles of A, at most
    int64_t counters, norm, d, e, x0, x1, xf, af, sa, sb, part, bytes;
};
constexpr int kPairs = 76;    // pairs of CTAs that the device holds

// One way of cutting, and what it takes: a product's stages one after the other, as often as its pieces go round the
// device, and what becomes of the last accumulator.  A stage takes 0.36 us on a pair's tile of 256 columns, 0.27 on one of
// 128, and 0.36 on a single CTA's, which is half of that work (the copies alone 0.30, 0.21 and 0.28).  An accumulator takes 4, 2
// and 1 us, and its splits' exchange 10.5, 6 and 5 and a quarter more for each split.  What comes on top of each product (3 us: the copies' latency, the
// barrier) is the same for all.
double cut(Plan& q, bool pair) {
    q.pair = pair;
    q.ctas = pair ? TileOf<true>::kCtas : TileOf<false>::kCtas;
    const int64_t rows = pair ? TileOf<true>::kRows : TileOf<false>::kRows, widest = pair ? TileOf<true>::kCols : TileOf<false>::kCols;
    const int64_t units = pair ? kPairs : 2 * kPairs;
    q.tm = al(q.m, rows) / rows;
    q.bm = q.tm * rows / kBox;
    q.bn = al(q.n, pair ? widest : 2 * kBox) / kBox;
    double all = 0.0;
    for (int k = 0; k < 3; ++k) {
        const int64_t depth = pair ? TileOf<true>::kDepth : TileOf<false>::kDepth, stages = (k == 0 ? q.bn : q.bm) / depth;
        double best = -1.0;
        for (int64_t cols = widest; cols >= (pair ? 128 : 64); cols /= 2) {
            const double stage = !pair ? 0.36 : cols == 256 ? 0.36 : 0.27, exchange = !pair ? 5.0 : cols == 256 ? 10.5 : 6.0;
            const int64_t tiles = q.batch * (k == 2 ? q.tm * (q.bn * kBox / cols) : q.tm * (q.tm + 1) / 2 * (rows / cols));
            const int64_t most = k == 2 || tiles >= units ? 1 : units / tiles;
            for (int64_t s = 1; s <= most && s <= stages && s <= 32; ++s) {
                const int64_t per = (stages + s - 1) / s;
                const double t = double((tiles * s + units - 1) / units * per) * stage + (s > 1 ? exchange + 0.25 * double(s) : double(cols) / 64.0);
                if (best >= 0.0 && t >= best) continue;
                best = t;
                q.cols[k] = cols;
                q.splits[k] = (stages + per - 1) / per;
                q.tiles[k] = tiles;
                q.items[k] = tiles * q.splits[k];
            }
        }
        all += best;
    }
    return all;
}

// (of one matrix at least)
Plan plan_of(int64_t batch, int64_t rows, int64_t cols) {
    Plan q{}, single{};
    q.batch = batch;
    q.turned = rows > cols;
    q.m = q.turned ? cols : rows;
    q.n = q.turned ? rows : cols;
    single = q;
    if (cut(single, false) <= cut(q, true)) q = single;
    q.parts = al(q.m * q.n, 4096) / 4096;
    if (q.parts > kNormCtas) q.parts = kNormCtas;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += al(bytes, 256);
        return here;
    };
    const int64_t x = batch * q.bm * q.bn * kBoxBytes, sq = batch * q.bm * q.bm * kBoxBytes, diag = batch * q.bm * kBox * 4;
    int64_t part = 0;
    for (int k = 0; k < 2; ++k) {
        const int64_t sums = q.splits[k] > 1 ? q.items[k] * q.ctas * kCtaRows * q.cols[k] : 0;
        part = sums > part ? sums : part;
    }
    q.half = q.tiles[0] > q.tiles[1] ? q.tiles[0] : q.tiles[1];
    q.counters = take((1 + 2 * q.half * q.ctas) * 4);
    q.norm = take(batch * q.parts * 16);
    q.d = take(diag);
    q.e = take(diag);
    q.x0 = take(x);
    q.x1 = take(x);
    q.xf = take(2 * x);
    q.af = take(2 * sq);
    q.sa = take(sq);
    q.sb = take(sq);
    q.part = take(part * 4);
    q.bytes = at;
    return q;
}

// Largest magnitude of y -> a y + b y^3 + c y^5 on [0, r], and of b y^2 + c y^4.
double most_of(double a, double b, double c, double r) {
    auto f = [&](double y2) { return std::fabs(std::sqrt(y2) * (a + y2 * (b + y2 * c))); };
    double most = f(r * r);
    // a + 3 b y^2 + 5 c y^4 = 0
    const double disc = 9 * b * b - 20 * a * c;
    if (disc >= 0)
        for (double s : {-1.0, 1.0}) {
            const double y2 = c != 0 ? (-3 * b + s * std::sqrt(disc)) / (10 * c) : b != 0 ? -a / (3 * b) : -1.0;
            if (y2 > 0 && y2 < r * r) most = std::fmax(most, f(y2));
        }
    return most;
}
double most_of_b(double b, double c, double r) {
    auto f = [&](double y2) { return std::fabs(y2 * (b + y2 * c)); };
    double most = f(r * r);
    if (c != 0 && -b / (2 * c) > 0 && -b / (2 * c) < r * r) most = std::fmax(most, f(-b / (2 * c)));
    return most;
}
// The largest power of two that takes `most` to no more than half of fp16's range.
float room_for(double most) {
    int k = 0;
    std::frexp(32768.0 / std::fmax(most, 1.0), &k);
    return float(std::ldexp(1.0, k - 1 > 15 ? 15 : k - 1));
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
    static EncodeFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<EncodeFn>(f);
    }();
    return fn;
}
// Maps of `rows` x `cols` boxes (with two each way, where there are two).
bool encode(BoxMaps* maps, void* p, int64_t rows, int64_t cols) {
    const EncodeFn fn = encode_fn();
    if (!fn || rows > INT32_MAX || cols > INT32_MAX) return false;
    const cuuint64_t dims[4] = {kBox, kBox, cuuint64_t(cols), cuuint64_t(rows)};
    const cuuint64_t strides[3] = {kBox * 2, kBoxBytes, cuuint64_t(cols) * kBoxBytes};
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    auto one = [&](CUtensorMap* map, cuuint32_t across, cuuint32_t down) {
        const cuuint32_t box[4] = {kBox, kBox, across, down};
        return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, p, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
    };
    return one(&maps->down, 1, 2) && one(&maps->beside, 2, 1) && one(&maps->one, 1, 1);
}

template <bool PAIR>
cudaError_t resident(int device, int* n) {
    static int held[kOpsMaxDevices];
    if (!held[device]) {
        cudaError_t e = cudaFuncSetAttribute(orth_product_kernel<PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, TileOf<PAIR>::kSmem);
        if (e != cudaSuccess) return e;
        int k = 0;
        if (PAIR) {
            cudaLaunchAttribute attr{};
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = 2;
            attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cudaLaunchConfig_t c{};
            c.gridDim = dim3(2 * kPairs);
            c.blockDim = dim3(kThreads);
            c.dynamicSmemBytes = TileOf<PAIR>::kSmem;
            c.attrs = &attr;
            c.numAttrs = 1;
            e = cudaOccupancyMaxActiveClusters(&k, orth_product_kernel<PAIR>, &c);
        } else {
            e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&k, orth_product_kernel<PAIR>, kThreads, TileOf<PAIR>::kSmem);
            k *= ops_sm_count(device);
        }
        if (e != cudaSuccess) return e;
        if (k < 1) return cudaErrorCooperativeLaunchTooLarge;
        held[device] = k;
    }
    *n = held[device];
    return cudaSuccess;
}

template <bool PAIR>
cudaError_t launch_products(int device, OrthParams& p, const Plan& q, cudaStream_t s) {
    int units = 0;
    cudaError_t e = resident<PAIR>(device, &units);
    if (e != cudaSuccess) return e;
    int64_t want = 1;
    for (int k = 0; k < 3; ++k) {
        int64_t items = q.items[k];
        // splits wait for one another, so each needs a CTA of its own
        if (p.splits[k] > 1 && items > units) {
            items /= p.splits[k];
            p.splits[k] = 1;
        }
        want = items > want ? items : want;
    }
    if (want < units) units = int(want);
    cudaLaunchAttribute attr[2] = {};
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(unsigned(units * q.ctas));
    c.blockDim = dim3(kThreads);
    c.dynamicSmemBytes = TileOf<PAIR>::kSmem;
    c.stream = s;
    c.attrs = attr;
    c.numAttrs = PAIR ? 2 : 1;
    OrthMaps maps;
    const int64_t boxes = q.batch * q.bm;
    if (!encode(&maps.x[0], p.x[0], boxes, q.bn) || !encode(&maps.x[1], p.x[1], boxes, q.bn) || !encode(&maps.sa, p.sa, boxes, q.bm) ||
        !encode(&maps.sb, p.sb, boxes, q.bm))
        return cudaErrorInvalidValue;
    cudaGetLastError();
    return cudaLaunchKernelEx(&c, orth_product_kernel<PAIR>, maps, p);
}

// CTAs and columns over 64 of each that a small matrix takes (0: it is not one).
struct Small {
    int ctas, blocks;
};
// As few as hold it; twice as many, with half of the columns each, where the device has room for all matrices' clusters at once (128 x
// 512: 39 us with four, 43 with two; 128 x 1024 42 with eight, 47 with four, but sixteen of them 84 and 49).
Small small_of(int64_t batch, int64_t m, int64_t n) {
    if (m > kSmallRows || n > kSmallCols * kSmallCtas) return {0, 0};
    int c = 1;
    while (int64_t(c) * kSmallCols < n) c *= 2;
    if (c > 1 && c < kSmallCtas && batch * 2 * c <= (c > 2 ? 64 : 128)) c *= 2;
    return {c, int((n + c * 64 - 1) / (c * 64))};
}
template <int K>
cudaError_t launch_small(const SmallParams& p, int64_t batch, cudaStream_t s) {
    static bool ready[kOpsMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && !ready[dev]) {
        e = cudaFuncSetAttribute(orth_small_kernel<K>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallSmem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(orth_small_kernel<K>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        ready[dev] = e == cudaSuccess;
    }
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = unsigned(p.ctas);
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(unsigned(batch * p.ctas));
    c.blockDim = dim3(kSmallThreads);
    c.dynamicSmemBytes = kSmallSmem;
    c.stream = s;
    c.attrs = &attr;
    c.numAttrs = 1;
    cudaGetLastError();
    return cudaLaunchKernelEx(&c, orth_small_kernel<K>, p);
}

// Checks of one array of matrices; the whole of it as one span.
lc_status check_mats(const char* call, const char* name, const lc_mats* a, int64_t batch, int64_t rows, int64_t cols, bool out,
                     Span2* span) {
    if (!a) return fail_status(LC_ERR_INVALID_ARG, "%s: %s is NULL", call, name);
    const int e = elem_size(a->dtype);
    if (!e) return fail_status(LC_ERR_INVALID_ARG, "%s: %s has unknown dtype %d", call, name, int(a->dtype));
    if (reinterpret_cast<uintptr_t>(a->data) % uintptr_t(e))
        return fail_status(LC_ERR_INVALID_ARG, "%s: %s is not element-aligned", call, name);
    constexpr int64_t kFar = int64_t(1) << 40;
    if (a->stride < 0 || a->batch_stride < 0 || a->stride > kFar || a->batch_stride > kFar)
        return fail_status(LC_ERR_INVALID_ARG, "%s: %s has strides %lld and %lld", call, name, (long long)a->batch_stride,
                           (long long)a->stride);
    // an output's rows do not meet: matrix after matrix, or row after row of all of them
    const int64_t st = rows > 1 ? a->stride : 0, bs = batch > 1 ? a->batch_stride : 0;
    if (out && !((rows == 1 || st >= cols) && (batch <= 1 || bs >= (rows - 1) * st + cols)) &&
        !((batch <= 1 || bs >= cols) && (rows == 1 || st >= (batch - 1) * bs + cols)))
        return fail_status(LC_ERR_INVALID_ARG, "%s: rows of %s overlap (strides %lld and %lld)", call, name,
                           (long long)a->batch_stride, (long long)a->stride);
    *span = {name, a->data, batch > 0 ? 1 : 0, ((batch - 1) * bs + (rows - 1) * st + cols) * e, 0, out};
    return LC_OK;
}

bool rows_wide(const void* p, int64_t pitch, int64_t batch_pitch) { return aligned16(p) && pitch % 16 == 0 && batch_pitch % 16 == 0; }

bool orth_sizes(int64_t batch, int64_t rows, int64_t cols) {
    return batch >= 0 && batch <= 65535 && rows > 0 && cols > 0 && rows <= LC_ORTH_MAX_DIM && cols <= LC_ORTH_MAX_DIM &&
           batch * ((rows + 127) / 128) * ((cols + 127) / 128) < (int64_t(1) << 30);
}

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" uint64_t lc_orthogonalize_workspace(int64_t batch, int64_t rows, int64_t cols) {
    if (!orth_sizes(batch, rows, cols) || batch == 0) return 0;
    if (small_of(batch, rows < cols ? rows : cols, rows < cols ? cols : rows).ctas) return 0;
    return uint64_t(plan_of(batch, rows, cols).bytes);
}

extern "C" lc_status lc_orthogonalize(int device, void* cuda_stream, const lc_mats* update, int64_t batch, int64_t rows,
                                      int64_t cols, const lc_mats* momentum, double beta, int32_t nesterov, int32_t steps,
                                      const double* coefficients, double eps, const lc_mats* out, void* workspace,
                                      uint64_t workspace_bytes) {
    const char* call = "lc_orthogonalize";
    set_last_error("");
    if (!orth_sizes(batch, rows, cols))
        return fail_status(LC_ERR_INVALID_ARG, "%s: %lld matrices of %lld x %lld (at most LC_ORTH_MAX_DIM = %d a side)", call,
                           (long long)batch, (long long)rows, (long long)cols, LC_ORTH_MAX_DIM);
    if (steps < 1 || steps > kMaxSteps || !coefficients)
        return fail_status(LC_ERR_INVALID_ARG, "%s: 1 to %d steps with three coefficients each are needed", call, kMaxSteps);
    if (!(eps >= 0.0) || eps > 1e30) return fail_status(LC_ERR_INVALID_ARG, "%s: eps %g", call, eps);
    if (momentum && !(beta >= 0.0 && beta < 1.0)) return fail_status(LC_ERR_INVALID_ARG, "%s: beta %g", call, beta);
    Span2 spans[4];
    int n = 0;
    lc_status st = check_mats(call, "update", update, batch, rows, cols, false, &spans[n++]);
    if (st == LC_OK && momentum) st = check_mats(call, "momentum", momentum, batch, rows, cols, true, &spans[n++]);
    if (st == LC_OK) st = check_mats(call, "out", out, batch, rows, cols, true, &spans[n++]);
    if (st != LC_OK) return st;
    if (momentum && momentum->dtype != LC_F32) return fail_status(LC_ERR_INVALID_ARG, "%s: the momentum is kept in fp32", call);
    if (out->dtype != LC_BF16) return fail_status(LC_ERR_INVALID_ARG, "%s: out is bf16", call);
    const int64_t m = rows < cols ? rows : cols, long_side = rows < cols ? cols : rows;
    // what no singular value exceeds at any step, from which the operands' scales follow
    OrthParams p{};
    double r = 1.0, most = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double a = coefficients[3 * k], b = coefficients[3 * k + 1], c = coefficients[3 * k + 2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c) || std::fabs(a) > 1e3 || std::fabs(b) > 1e3 || std::fabs(c) > 1e3)
            return fail_status(LC_ERR_INVALID_ARG, "%s: coefficients %g, %g, %g", call, a, b, c);
        const double in_b = most_of_b(b, c, r);
        p.step[k] = {float(a), float(b), float(c), room_for(in_b)};
        r = most_of(a, b, c, r);
        if (!(r <= 16.0) || in_b > 16384.0)
            return fail_status(LC_ERR_INVALID_ARG, "%s: the coefficients of step %d let singular values grow to %g", call, k, r);
        most = std::fmax(most, r);
    }
    p.a_scale = room_for(most * most);
    p.x_scale = room_for(most);
    // elements of about 1 where the matrix has no structure: sqrt(m n) times those of X
    const float middle = float(std::ldexp(1.0, std::ilogb(std::sqrt(double(m) * double(long_side)))));
    if (middle < p.x_scale) p.x_scale = middle;
    const uint64_t need = lc_orthogonalize_workspace(batch, rows, cols);
    if (workspace_bytes < need)
        return fail_status(LC_ERR_CAPACITY, "%s: %llu bytes of workspace, %llu needed", call, (unsigned long long)workspace_bytes,
                           (unsigned long long)need);
    if (need && reinterpret_cast<uintptr_t>(workspace) % 256)
        return fail_status(LC_ERR_INVALID_ARG, "%s: the workspace is not 256-byte aligned", call);
    OnDevice cur(device);
    spans[n++] = {"workspace", workspace, need ? 1 : 0, int64_t(need), 0, true};
    st = ops_check(call, device, spans, n);
    if (st != LC_OK) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "%s: cannot make device %d current", call, device);
    if (!batch) return LC_OK;
    const Plan q = plan_of(batch, rows, cols);
    const Small small = small_of(batch, m, long_side);
    uint8_t* const w = static_cast<uint8_t*>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    PrepParams a{};
    const int ue = elem_size(update->dtype);
    a.u = static_cast<const uint8_t*>(update->data);
    a.u_pitch = update->stride * ue;
    a.u_batch = update->batch_stride * ue;
    a.wide = rows_wide(a.u, rows > 1 ? a.u_pitch : 0, batch > 1 ? a.u_batch : 0);
    if (momentum) {
        a.m = static_cast<uint8_t*>(momentum->data);
        a.m_pitch = momentum->stride * 4;
        a.m_batch = momentum->batch_stride * 4;
        a.wide = a.wide && rows_wide(a.m, rows > 1 ? a.m_pitch : 0, batch > 1 ? a.m_batch : 0);
    }
    a.part = reinterpret_cast<float4*>(w + q.norm);
    a.zero = reinterpret_cast<uint32_t*>(w + q.counters);
    a.nzero = int32_t((q.norm - q.counters) / 4);
    a.parts = int32_t(q.parts);
    a.hi = w + q.x0;
    a.xf = w + q.xf;
    a.rows = rows;
    a.cols = cols;
    a.beta = float(beta);
    a.x_scale = p.x_scale;
    a.eps = eps;
    a.u_bf16 = update->dtype == LC_BF16;
    a.nesterov = nesterov != 0;
    a.turned = q.turned;
    a.bm = int32_t(q.bm);
    a.bn = int32_t(q.bn);
    if (small.ctas) {
        SmallParams o{};
        o.u = a.u;
        o.u_pitch = a.u_pitch;
        o.u_batch = a.u_batch;
        o.m = a.m;
        o.m_pitch = a.m_pitch;
        o.m_batch = a.m_batch;
        o.out = static_cast<uint8_t*>(out->data);
        o.out_pitch = out->stride * 2;
        o.out_batch = out->batch_stride * 2;
        o.rows = rows;
        o.cols = cols;
        o.eps = eps;
        o.beta = float(beta);
        o.x_scale = p.x_scale;
        o.a_scale = p.a_scale;
        o.ctas = small.ctas;
        o.u_bf16 = a.u_bf16;
        o.nesterov = a.nesterov;
        o.turned = a.turned;
        o.steps = steps;
        o.stall = ops_stall();
        o.wide = a.wide;
        o.out_wide = rows_wide(o.out, rows > 1 ? o.out_pitch : 0, batch > 1 ? o.out_batch : 0);
        for (int k = 0; k < steps; ++k) o.step[k] = p.step[k];
        cudaError_t (*const launch[])(const SmallParams&, int64_t, cudaStream_t) = {launch_small<1>, launch_small<2>, launch_small<3>,
                                                                                   launch_small<4>};
        return ops_launched(call, launch[small.blocks - 1](o, batch, s));
    }
    PrepParams flat = a;
    if (update->stride == cols && (!momentum || momentum->stride == cols)) {
        flat.rows = 1;
        flat.cols = rows * cols;
        flat.wide = rows_wide(a.u, 0, batch > 1 ? a.u_batch : 0) && (!momentum || rows_wide(a.m, 0, batch > 1 ? a.m_batch : 0));
    }
    cudaGetLastError();
    orth_norm_kernel<<<dim3(unsigned(q.parts), unsigned(batch)), 256, 0, s>>>(flat);
    cudaError_t err = cudaGetLastError();
    if (err != cudaSuccess) return ops_launched(call, err);
    const int64_t boxes = q.bm * q.bn, most_ctas = int64_t(ops_sm_count(device)) * 8;
    orth_split_kernel<<<dim3(unsigned(boxes < most_ctas ? boxes : most_ctas), unsigned(batch)), 256, 0, s>>>(a);
    err = cudaGetLastError();
    if (err != cudaSuccess) return ops_launched(call, err);
    p.count = reinterpret_cast<uint32_t*>(w + q.counters);
    p.arrived = p.count + 1;
    p.d = reinterpret_cast<float*>(w + q.d);
    p.e = reinterpret_cast<float*>(w + q.e);
    p.x[0] = w + q.x0;
    p.x[1] = w + q.x1;
    p.xf = w + q.xf;
    p.af = w + q.af;
    p.sa = w + q.sa;
    p.sb = w + q.sb;
    p.part = reinterpret_cast<float*>(w + q.part);
    p.out = static_cast<uint8_t*>(out->data);
    p.out_pitch = out->stride * 2;
    p.out_batch = out->batch_stride * 2;
    // the last CTAs start once other streams' kernels make room for them, and a product takes its time (at a twentieth of the
    // tensor cores' rate)
    p.limit_ns = (ops_stall() ? kWaitNs : 20 * kWaitNs) + uint64_t(2.0 * double(batch) * double(q.m) * double(q.m) * double(q.n) * 1e-5);
    p.batch = int32_t(batch);
    p.m = int32_t(q.m);
    p.n = int32_t(q.n);
    p.bm = int32_t(q.bm);
    p.bn = int32_t(q.bn);
    p.steps = steps;
    p.tiles = int32_t(q.half);
    for (int k = 0; k < 3; ++k) {
        p.splits[k] = int32_t(q.splits[k]);
        p.cols[k] = int32_t(q.cols[k]);
    }
    p.turned = q.turned;
    p.wide = rows_wide(p.out, rows > 1 ? p.out_pitch : 0, batch > 1 ? p.out_batch : 0);
    p.stall = ops_stall();
    err = q.pair ? launch_products<true>(device, p, q, s) : launch_products<false>(device, p, q, s);
    return ops_launched(call, err);
}
