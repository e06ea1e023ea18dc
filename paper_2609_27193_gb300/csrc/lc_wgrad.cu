// lc_wgrad.cu -- the weight gradient of a linear layer whose input was kept in 8
// bits: dw[n][k] = sum over t of dy[t][n] * q[t][k] * 2^e[t][k / 128].
//
// A matrix product over the tokens on the 5th-generation tensor cores.  A value of
// the checkpoint is exactly a bf16 number, so it is an operand without a rounding;
// it is made on the way and never leaves the multiprocessor.  Two CTAs of a
// cluster share a tile of 256 features x 256 columns of dy: each holds 128 of
// either, so a byte of dy that comes from L2 serves 256 features.  In each CTA
//
//   warp 0    one thread issues the bulk tensor copies of a stage (64 tokens): an
//             8-bit tile of the checkpoint, a bf16 tile of dy
//   warp 1    one thread of the first CTA issues the products for both
//   warps 2-3 bring the tokens' exponents, kChunk stages ahead at a time
//   warps 4-11 turn the 8-bit tile into the bf16 operand in shared memory, four
//             warps a stage; tokens are rows there as in memory, and the product
//             takes both operands that way, so nothing is transposed
//   warps 12-19 add up the results
//
// The tensor cores add in fp32, but a chain of many products loses more than a sum
// in registers does (8192 tokens in one chain: 2.5e-6 off; in pieces of 1024:
// 1.9e-7).  So a chain is kChunk stages long; two accumulators in tensor memory
// take turns, and the last eight warps add the finished one to their registers
// while the other is being filled.  The CTAs are persistent and the stages of one
// tile follow those of the last, so the outputs are written while the next tile's
// products run.
//
// A 32-bit dy is split into three bf16 parts that add up to it (8 + 8 + 8 bits of
// significand, cut off, not rounded, so nothing overflows; exactly, but for bits below
// bf16's least 2^-133, which only values below 2^-110 have); a stage then has the tiles
// of all three, and the operand is made once for them.  That and a bf16 dy
// off 16-byte boundaries go into aligned rows in the workspace, by a kernel of their
// own.  Few output tiles are split over the tokens; the parts are
// added in order by another kernel.
//
// Waits are bounded: one that runs out leaves NaN in the outputs.
#include <cuda.h>

#include "lc_bulk.cuh"
#include "lc_ops.cuh"

namespace lc {
namespace {

constexpr int kHalf = 128;       // features and columns of dy that a CTA of the pair holds
constexpr int kTile = 2 * kHalf; // of the pair's tile
constexpr int kTok = 64;         // tokens of a stage
constexpr int kXBytes = kTok * kHalf;              // 8-bit tile
constexpr int kBox = 64;                           // columns of a copy or operand box: 128 bytes, the swizzle's span
constexpr int kBoxBytes = kTok * kBox * 2;
constexpr int kOpBytes = kHalf / kBox * kBoxBytes; // a bf16 tile
// A stage holds the tiles of all parts of dy (one, or three of a 32-bit dy), the
// 8-bit tile and the operand made of it, once for all parts.
template <int PARTS>
struct StageOf {
    static constexpr int kLoad = PARTS * kOpBytes + kXBytes;    // what its copies bring
    static constexpr int kBytes = kLoad + kOpBytes;
    static constexpr int kStages = PARTS == 1 ? 5 : 3;          // as many as fit
    // stages that one accumulator adds up.  Three parts are added to it one by one, the smaller ones to sums of the
    // larger: 2047 tokens are 1.0e-6 off in chains of 5 stages, 5.8e-7 in chains of 2
    static constexpr int kChunk = PARTS == 1 ? 16 : 2;
    static constexpr int kSmem = kStages * kBytes + 1024;       // and room to align the tiles to 1024 bytes
};
constexpr int kConvWarp = 4, kConvWarps = 8;       // first converter warp (a multiple of 4), their number
constexpr int kSumWarp = kConvWarp + kConvWarps, kSumWarps = 8;
constexpr int kThreads = (kSumWarp + kSumWarps) * 32;
// Registers of a thread once the roles part: 4 * 32 * 40 + 8 * 32 * 56 + 8 * 32 * 160 = 60416, within the 640 * 96 =
// 61440 of the launch.
constexpr int kLaunchRegs = 96, kRoleRegs = 40, kConvRegs = 56, kSumRegs = 160;
static_assert(kConvWarp * 32 * kRoleRegs + kConvWarps * 32 * kConvRegs + kSumWarps * 32 * kSumRegs <= kThreads * kLaunchRegs &&
                  kThreads * kLaunchRegs <= 65536, "registers");
constexpr int kTmemCols = 512;                     // two accumulators of 256 columns
constexpr int kAcc = kTile / 2;                    // columns that a thread adds up

// Instruction descriptor: fp32 accumulator, bf16 operands, both with their rows
// along the reduction; 256 x 256.
constexpr uint32_t kIdesc = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | uint32_t(kTile / 8) << 17 | uint32_t(kTile / 16) << 24;

struct WgradParams {
    const int8_t* e;
    uint8_t* dw;
    float* part;           // [splits][rows][dim] (splits > 1)
    int64_t e_pitch, dw_pitch;
    int32_t ntok, rows, dim;
    int32_t items;         // tiles * splits
    int32_t ntiles_n, stages, splits, per_split;   // stages in all, of a split
    int32_t tok_part;      // rows of dy between the parts
    int32_t dw_bf16;
    int32_t stall;         // test switch: the second CTA's first copy announces 16 bytes that never come
};

__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

// Once the products issued so far are done: an arrival at the barrier in both CTAs.
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
        "h"(uint16_t(3))
        : "memory");
}

// d += a * b over both CTAs' halves; both operands in shared memory.
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
}

// Shared-memory descriptor of a bf16 tile: 64-column boxes of 128-byte swizzled
// rows, 8 tokens 1024 bytes apart, the next 64 columns a box further.
__device__ __forceinline__ uint64_t op_desc(uint32_t addr) {
    return uint64_t((addr & 0x3ffffu) >> 4) | uint64_t(kBoxBytes >> 4) << 16 | uint64_t(1024 >> 4) << 32 |
           uint64_t(1) << 46 | uint64_t(2) << 61;
}

__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
}

// The barrier at this address in the pair's first CTA.
__device__ __forceinline__ uint32_t in_first(uint32_t bar) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(bar));
    return r;
}
// An arrival at a barrier of either CTA.  What it announces is read where it was
// written (the tensor core of each multiprocessor reads its own shared memory, after
// a proxy fence there), so no memory has to become visible to the other CTA: a
// release for the whole cluster costs a full memory barrier a stage, which took most
// of the converters' time (the kernel 1.36 ms instead of 0.82 at 8192 tokens, 14336 ->
// 4096).
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Bytes 0 and 2 of a word make one pair and bytes 1 and 3 the other, which spares
// the permutations that neighbours would need: of every four features of the
// operand the middle two have changed places.
__device__ __forceinline__ int feature_of(int row) { return (row & ~3) | (row & 1) << 1 | (row >> 1 & 1); }

// One piece of work: a tile, or a split of one.
struct Item {
    int n0, k0, split, s0, stages;
};
__device__ __forceinline__ Item item_of(const WgradParams& p, int i) {
    Item w;
    const int tile = i / p.splits;
    w.split = i - tile * p.splits;
    w.n0 = tile % p.ntiles_n * kTile;
    w.k0 = tile / p.ntiles_n * kTile;
    w.s0 = w.split * p.per_split;
    w.stages = (w.s0 + p.per_split < p.stages ? w.s0 + p.per_split : p.stages) - w.s0;
    return w;
}

template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// A place in a ring of N and the parity of its round.
template <int N>
struct Ring {
    int at = 0;
    uint32_t round = 0;   // parity
    __device__ __forceinline__ void next() {
        if (++at == N) {
            at = 0;
            round ^= 1;
        }
    }
};

// ACC: the outputs are added to (never with splits).
template <int PARTS, bool ACC>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    wgrad_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap ymap, WgradParams p) {
    constexpr int kStages = StageOf<PARTS>::kStages, kChunk = StageOf<PARTS>::kChunk;
    constexpr int kStageBytes = StageOf<PARTS>::kBytes, kLoadBytes = StageOf<PARTS>::kLoad;
    extern __shared__ uint8_t raw[];
    // full and empty: a stage's copies have landed / its products are done (each CTA's own).  converted: both CTAs'
    // operands are in place (the first CTA's).  summed: an accumulator is complete; taken: both CTAs have read it (the
    // first CTA's).  scaled and used: a chunk's scales are there / no longer needed.
    __shared__ __align__(8) uint64_t bars[3 * kStages + 8];
    __shared__ __align__(16) uint16_t scales[2][kChunk * kTok];   // 2^e as bf16
    __shared__ uint32_t tmem_base;
    __shared__ volatile uint32_t failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x & 1, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const uint32_t tiles = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, converted = empty + 8 * kStages;
    const uint32_t summed = converted + 8 * kStages, taken = summed + 16, scaled = taken + 16, used = scaled + 16;
    dependents_may_start();
    if (threadIdx.x == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&xmap) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&ymap) : "memory");
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
            mbar_init(converted + 8 * i, kConvWarps);   // half of each CTA's
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(summed + 8 * i, 1);
            mbar_init(taken + 8 * i, 2 * kSumWarps);
            mbar_init(scaled + 8 * i, 2);
            mbar_init(used + 8 * i, kConvWarps);
        }
        failed = 0;
        mbar_init_fence();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_barrier();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    dependency_wait();

    if (warp < kConvWarp) {
        fewer_registers<kRoleRegs>();
        bool ok = true;
        if (warp == 0 && lane == 0) {
            Ring<kStages> st;
            int it = 0;
            for (int i = pair; i < p.items && ok; i += pairs) {
                const Item w = item_of(p, i);
                int t = w.s0 * kTok;
                for (int s = 0; s < w.stages; ++s, ++it, st.next()) {
                    ok = it < kStages || mbar_wait_bounded(empty + 8 * st.at, st.round ^ 1, kWaitNs);
                    if (!ok) break;
                    const uint32_t at = tiles + st.at * kStageBytes, bar = full + 8 * st.at;
                    mbar_expect_tx(bar, kLoadBytes + (it == 0 && rank == 1 && p.stall ? 16 : 0));
                    tma_2d(at + PARTS * kOpBytes, &xmap, w.k0 + rank * kHalf, t, bar);
#pragma unroll
                    for (int part = 0; part < PARTS; ++part)
                        for (int j = 0; j < kHalf / kBox; ++j)
                            tma_2d(at + part * kOpBytes + j * kBoxBytes, &ymap, w.n0 + rank * kHalf + j * kBox, part * p.tok_part + t, bar);
                    t += kTok;
                }
            }
            // every copy lands before the CTA's memory is given back
            for (int i = it > kStages ? it - kStages : 0; i < it; ++i)
                if (!mbar_wait_bounded(full + 8 * (i % kStages), (i / kStages) & 1, kWaitNs)) ok = false;
            // and so does every arrival that ends a stage's products: they come to both CTAs of the pair, and nobody else
            // waits for the last round of them.  (Where products are missing one wait runs out, long after the arrivals
            // of those there are.)
            bool ended = true;
            for (int i = it > kStages ? it - kStages : 0; i < it && ended; ++i)
                ended = mbar_wait_bounded(empty + 8 * (i % kStages), (i / kStages) & 1, kWaitNs);
            ok = ok && ended;
        } else if (warp == 1 && lane == 0 && rank == 0) {
            Ring<kStages> st;
            Ring<2> acc;
            int chunk = 0;
            for (int i = pair; i < p.items && ok; i += pairs) {
                const Item w = item_of(p, i);
                for (int s = 0; s < w.stages; ++s, st.next()) {
                    const bool first = s % kChunk == 0;
                    if (first && chunk >= 2) ok = mbar_wait_bounded(taken + 8 * acc.at, acc.round ^ 1, kWaitNs);
                    ok = ok && mbar_wait_bounded(converted + 8 * st.at, st.round, kWaitNs);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t y = op_desc(tiles + st.at * kStageBytes), x = y + (kLoadBytes >> 4);
                    // 16 tokens are 2048 bytes further
#pragma unroll
                    for (int part = 0; part < PARTS; ++part)
#pragma unroll
                        for (int k = 0; k < kTok / 16; ++k)
                            tc_mma(tmem + acc.at * kTile, x + k * (2048 >> 4), y + part * (kOpBytes >> 4) + k * (2048 >> 4), kIdesc,
                                   !first || part > 0 || k > 0);
                    tc_commit(empty + 8 * st.at);
                    if (s % kChunk == kChunk - 1 || s == w.stages - 1) {
                        tc_commit(summed + 8 * acc.at);
                        acc.next();
                        ++chunk;
                    }
                }
            }
        } else if (warp >= 2) {
            int chunk = 0;
            for (int i = pair; i < p.items && ok; i += pairs) {
                const Item w = item_of(p, i);
                const int f = w.k0 + rank * kHalf;
                const int8_t* ep = p.e + f / LC_ACT_BLOCK;
                for (int s = 0; s < w.stages; s += kChunk, ++chunk) {
                    const int buf = chunk & 1, t_in = (warp - 2) * 32 + lane;
                    int e[kChunk];
#pragma unroll
                    for (int j = 0; j < kChunk; ++j) {
                        const int t = (w.s0 + s + j) * kTok + t_in;
                        e[j] = s + j < w.stages && t < p.ntok && f < p.dim ? int(__ldg(ep + int64_t(t) * p.e_pitch)) : 0;
                    }
                    ok = chunk < 2 || mbar_wait_warp(used + 8 * buf, (chunk / 2 - 1) & 1);
                    if (!ok) break;
                    // the upper half of the fp32 number 2^e, NaN for 127
#pragma unroll
                    for (int j = 0; j < kChunk; ++j)
                        scales[buf][j * kTok + t_in] = e[j] == 127 ? uint16_t(0x7fff) : uint16_t((e[j] + 127) << 7);
                    mbar_arrive_warp(scaled + 8 * buf, lane);
                }
            }
        }
        if (!ok) failed = 1;
    } else if (warp < kSumWarp) {
        fewer_registers<kConvRegs>();
        const int group = (warp - kConvWarp) >> 2, w4 = warp & 3;
        // 16 features, the c-th of the 8-bit row's eight pieces, of tokens t0 + 4 r, r = 0..3.  They are pieces 2 (c mod 4)
        // and the next of the operand's row in box c / 4; piece i of token t lies at i xor (t mod 8).  Lanes of the second
        // box have the neighbour of the others' token, so eight lanes meet in no bank, neither here nor there.
        const int c = lane & 7, t0 = w4 * 16 + ((lane >> 3) ^ (c >> 2));
        const uint32_t x_off = PARTS * kOpBytes + t0 * kHalf + c * 16;
        const uint32_t row_off = kLoadBytes + (c >> 2) * kBoxBytes + t0 * 128, piece = uint32_t((c & 3) * 2 ^ (t0 & 7)) << 4;
        const uint32_t first_converted = in_first(converted);
        const uint32_t align = tiles - smem_addr(raw);
        Ring<kStages> st;
        bool ok = true;
        int it = 0, chunk = 0;
        for (int i = pair; i < p.items && ok; i += pairs) {
            const int stages = item_of(p, i).stages;
            for (int s = 0; s < stages; ++s, ++it, st.next()) {
                const int sb = chunk & 1;
                if (s % kChunk == 0) ok = mbar_wait_warp(scaled + 8 * sb, (chunk >> 1) & 1);
                if ((it & 1) == group && ok) {
                    // The rings are odd, so the other group had this place last, and a wait knows a round by its parity
                    // alone: where that copy landed later than this group's own ones since, the round before it would
                    // pass.  The place's last products come first: they are behind that copy, and this round's wait
                    // for this group.
                    ok = it < kStages || mbar_wait_warp(empty + 8 * st.at, st.round ^ 1);
                    ok = ok && mbar_wait_warp(full + 8 * st.at, st.round);
                    if (!ok) break;   // no arrival: the other CTA's products read this CTA's half of dy
                    const uint8_t* x = raw + align + st.at * kStageBytes + x_off;
                    uint4 q[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) q[r] = *reinterpret_cast<const uint4*>(x + r * 4 * kHalf);
                    // the stage's copies were issued after its last products: the operand's place is free
                    uint8_t* o = raw + align + st.at * kStageBytes + row_off;
                    const uint16_t* sc = &scales[sb][s % kChunk * kTok + t0];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint32_t s2 = sc[4 * r] * 0x10001u;
                        const uint32_t qw[4] = {q[r].x, q[r].y, q[r].z, q[r].w};
                        uint32_t v[8];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            v[2 * j] = act_pair(qw[j], s2);
                            v[2 * j + 1] = act_pair(qw[j] >> 8, s2);
                        }
                        const uint32_t at = piece ^ (r & 1) << 6;
                        *reinterpret_cast<uint4*>(o + r * 512 + at) = make_uint4(v[0], v[1], v[2], v[3]);
                        *reinterpret_cast<uint4*>(o + r * 512 + (at ^ 16)) = make_uint4(v[4], v[5], v[6], v[7]);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) arrive_cluster(first_converted + 8 * st.at);
                }
                if (!ok) break;
                if (s % kChunk == kChunk - 1 || s == stages - 1) {
                    mbar_arrive_warp(used + 8 * sb, lane);
                    ++chunk;
                }
            }
        }
        if (!ok) failed = 1;
    } else {
        more_registers<kSumRegs>();
        const int quad = warp & 3, half = (warp - kSumWarp) >> 2;
        const uint32_t first_taken = in_first(taken);
        const uint32_t from = tmem + (uint32_t(quad * 32) << 16) + half * kAcc;
        Ring<2> a;
        bool ok = true;
        for (int i = pair; i < p.items; i += pairs) {
            const Item w = item_of(p, i);
            float acc[kAcc];
#pragma unroll
            for (int j = 0; j < kAcc; ++j) acc[j] = 0.0f;
            for (int s = 0; s < w.stages && ok; s += kChunk, a.next()) {
                ok = mbar_wait_warp(summed + 8 * a.at, a.round);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int j = 0; j < kAcc; j += 16) {
                    uint32_t r[16];
                    tmem_ld16(from + a.at * kTile + j, r);
#pragma unroll
                    for (int k = 0; k < 16; ++k) acc[j + k] += __uint_as_float(r[k]);
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) arrive_cluster(first_taken + 8 * a.at);
            }
            if (!ok) failed = 1;
            const float off = failed ? __uint_as_float(0x7fffffffu) : 0.0f;   // NaN after a wait that ran out
            const int k = w.k0 + rank * kHalf + feature_of(quad * 32 + lane);
            const int n0 = w.n0 + half * kAcc;
            const int left = p.rows - n0, cnt = k < p.dim ? left : 0;
            // ACC and whole tiles have loops of their own: tests inside would make these unrolled loops twice as long,
            // and their instructions come from memory for a tile or two of few tokens (64 tokens, 4096 -> 4096 in bf16:
            // 27 us with the tests inside, 15 so)
            if (p.splits == 1 && p.dw_bf16) {
                // lanes two apart have neighbouring features: of two columns each takes one, with both features, so that
                // a store has 4 bytes (33 us with 2 bytes a store)
                const bool up = lane & 2;
                const int k2 = k & ~1;
                const bool second = k2 + 1 < p.dim;
                __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.dw + int64_t(n0 + (up ? 1 : 0)) * p.dw_pitch) + k2;
                const int64_t step = p.dw_pitch;           // two rows, in elements
                const bool wide = second && ((reinterpret_cast<uintptr_t>(o) | uintptr_t(p.dw_pitch)) & 3) == 0;
                auto pair = [&](int j, float& x, float& y) {
                    const float got = __shfl_xor_sync(0xffffffffu, up ? acc[j] : acc[j + 1], 2);
                    x = (up ? got : acc[j]) + off;
                    y = (up ? acc[j + 1] : got) + off;
                };
                if (__all_sync(0xffffffffu, wide && left >= kAcc)) {
#pragma unroll
                    for (int j = 0; j < kAcc; j += 2) {
                        float x, y;
                        pair(j, x, y);
                        uint32_t* at = reinterpret_cast<uint32_t*>(o);
                        if constexpr (ACC) {
                            const uint32_t old = *at;
                            x += __uint_as_float(old << 16);
                            y += __uint_as_float(old & 0xffff0000u);
                        }
                        *at = pack_bf16(x, y);
                        o += step;
                        asm volatile("" : "+l"(o)::"memory");   // one pointer that moves on, not kAcc of them
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < kAcc; j += 2) {
                        float x, y;
                        pair(j, x, y);
                        if (j + (up ? 1 : 0) < left && k2 < p.dim) {
                            o[0] = __float2bfloat16_rn(ACC ? __bfloat162float(o[0]) + x : x);
                            if (second) o[1] = __float2bfloat16_rn(ACC ? __bfloat162float(o[1]) + y : y);
                        }
                        o += step;
                        asm volatile("" : "+l"(o)::"memory");
                    }
                }
            } else {
                // (a split product leaves its parts here, and what is added to comes with their sum)
                float* o = p.splits > 1 ? p.part + (int64_t(w.split) * p.rows + n0) * p.dim + k
                                        : reinterpret_cast<float*>(p.dw + int64_t(n0) * p.dw_pitch) + k;
                const int64_t pitch = p.splits > 1 ? p.dim : p.dw_pitch / 4;
                if (__all_sync(0xffffffffu, cnt >= kAcc)) {
#pragma unroll
                    for (int j = 0; j < kAcc; ++j) {
                        *o = ACC ? *o + acc[j] + off : acc[j] + off;
                        o += pitch;
                        asm volatile("" : "+l"(o)::"memory");
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < kAcc; ++j) {
                        if (j < cnt) *o = ACC ? *o + acc[j] + off : acc[j] + off;
                        o += pitch;
                        asm volatile("" : "+l"(o)::"memory");
                    }
                }
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncwarp();
    __syncthreads();
    // the other CTA's barriers and operands are used until here
    cluster_barrier();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

struct StageParams {
    const uint8_t* dy;
    __nv_bfloat16* out;     // [parts][tokens padded][cols padded]
    int64_t dy_pitch, tok_pad, col_pad;
    int64_t ntok, rows;
    int32_t f32;
};

// dy into rows on 16-byte boundaries: a copy, or three bf16 parts that add up to a
// 32-bit value (bits below 2^-133 are lost).  Each part takes the next eight bits of the significand, cut off.
// An infinity or a NaN stays whole in the first part.
// A thread takes four columns of a row.
__global__ void __launch_bounds__(256) wgrad_stage_kernel(StageParams p) {
    dependents_may_start();
    const int64_t quads = p.col_pad / 4, n = p.tok_pad * p.col_pad;
    const int64_t item = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (item * 4 >= n) return;
    int64_t t, c;
    split_item(item, quads, t, c);
    c *= 4;
    const uint8_t* row = p.dy + t * p.dy_pitch;
    uint2* out = reinterpret_cast<uint2*>(p.out + item * 4);
    if (!p.f32) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = t < p.ntok && c + i < p.rows ? reinterpret_cast<const uint16_t*>(row)[c + i] : 0u;
        *out = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
        return;
    }
    float x[4];
    if (t < p.ntok && c + 4 <= p.rows && (reinterpret_cast<uintptr_t>(row) & 15) == 0) {
        const float4 v = *reinterpret_cast<const float4*>(row + c * 4);
        x[0] = v.x;
        x[1] = v.y;
        x[2] = v.z;
        x[3] = v.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = t < p.ntok && c + i < p.rows ? reinterpret_cast<const float*>(row)[c + i] : 0.0f;
    }
    uint32_t h[4];   // the upper half of what is left
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t bits = __float_as_uint(x[i]);
            if ((bits & 0x7f800000u) == 0x7f800000u) {
                // a NaN whose set bits are all cut off stays one
                h[i] = bits >> 16 | ((bits & 0x7fffffu) ? 0x40u : 0u);
                x[i] = 0.0f;
            } else {
                h[i] = bits >> 16;
                x[i] -= __uint_as_float(bits & 0xffff0000u);
            }
        }
        out[k * n / 4] = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
    }
}

struct JoinParams {
    const float* part;
    uint8_t* dw;
    int64_t dw_pitch, rows, dim;
    int32_t splits, accumulate, dw_bf16;
};

// A CTA takes 1024 columns of a row, four a thread.
__global__ void __launch_bounds__(256) wgrad_join_kernel(JoinParams p) {
    dependency_wait();
    const int64_t n = p.rows * p.dim;
    int64_t r, part;
    split_item(blockIdx.x, (p.dim + 1023) / 1024, r, part);
    const int64_t c0 = part * 1024 + threadIdx.x;
    const float* from = p.part + r * p.dim + c0;
    float s[4] = {};
#pragma unroll 4
    for (int k = 0; k < p.splits; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c0 + i * 256 < p.dim) s[i] += from[k * n + i * 256];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t c = c0 + i * 256;
        if (c >= p.dim) break;
        if (p.dw_bf16) {
            __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.dw + r * p.dw_pitch) + c;
            *o = __float2bfloat16_rn(p.accumulate ? __bfloat162float(*o) + s[i] : s[i]);
        } else {
            float* o = reinterpret_cast<float*>(p.dw + r * p.dw_pitch) + c;
            *o = p.accumulate ? *o + s[i] : s[i];
        }
    }
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

// A map of `rows` rows of `cols` elements, copied in boxes of box_cols x kTok.
bool encode(CUtensorMap* map, CUtensorMapDataType type, const void* p, int64_t cols, int64_t rows, int64_t pitch,
            int box_cols, CUtensorMapSwizzle swizzle) {
    const EncodeFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {cuuint64_t(cols), cuuint64_t(rows)};
    const cuuint64_t strides[1] = {cuuint64_t(pitch)};
    const cuuint32_t box[2] = {cuuint32_t(box_cols), cuuint32_t(kTok)};
    const cuuint32_t one[2] = {1, 1};
    return fn(map, type, 2, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int64_t al(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// How a product is cut: output tiles, parts of dy, and splits of the tokens where
// the tiles alone leave multiprocessors idle (each split at least 8 stages long: a
// stage takes half a microsecond, joining the parts four; 512 tokens of 256 -> 1024
// take 9.8 us in one split and 11.8 in two, 2047 of 2048 -> 512 with a 32-bit dy 37 us in
// one, 29 in two, 22.6 in four and 27 in eight).
constexpr int kPairs = 76;
struct Shape {
    int64_t tiles_n, tiles_k, stages, splits, per_split;
};
Shape shape_of(int64_t ntok, int64_t rows, int64_t dim, int32_t dy_dtype) {
    Shape s;
    s.tiles_n = (rows + kTile - 1) / kTile;
    s.tiles_k = (dim + kTile - 1) / kTile;
    s.stages = (ntok + kTok - 1) / kTok;
    const int64_t tiles = s.tiles_n * s.tiles_k;
    s.splits = tiles >= kPairs ? 1 : kPairs / tiles;
    const int64_t least = dy_dtype == LC_F32 ? 4 : 8;   // a stage of three parts takes twice as long
    if (s.splits > s.stages / least) s.splits = s.stages / least;
    if (s.splits < 1) s.splits = 1;
    s.per_split = (s.stages + s.splits - 1) / s.splits;
    s.splits = (s.stages + s.per_split - 1) / s.per_split;
    return s;
}
int64_t staged_bytes(int64_t ntok, int64_t rows, int32_t dy_dtype) {
    return al(al(ntok, kTok) * al(rows, 64) * 2 * (dy_dtype == LC_F32 ? 3 : 1), 256);
}
// The parts of split tokens lie at the workspace's start, a staged dy behind them.
int64_t part_bytes(const Shape& s, int64_t rows, int64_t dim) { return s.splits > 1 ? al(s.splits * rows * dim * 4, 256) : 0; }
// Whether dy has to be staged: 32 bits, or rows that a bulk tensor copy cannot take.
bool staged_dy(const lc_rows* dy, int64_t rows) {
    const int64_t pitch = dy->stride * elem_size(dy->dtype);
    return dy->dtype == LC_F32 || !aligned16(dy->data) || pitch % 16 || pitch < rows * 2;
}
// Pairs of CTAs that the device holds at once.
template <int PARTS, bool ACC>
cudaError_t resident_pairs(int device, int* pairs) {
    static int held[kOpsMaxDevices];
    constexpr int kSmem = StageOf<PARTS>::kSmem;
    if (!held[device]) {
        cudaError_t e = cudaFuncSetAttribute(wgrad_kernel<PARTS, ACC>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return e;
        cudaLaunchAttribute attr{};
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 2;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cudaLaunchConfig_t c{};
        c.gridDim = dim3(2 * kPairs);
        c.blockDim = dim3(kThreads);
        c.dynamicSmemBytes = kSmem;
        c.attrs = &attr;
        c.numAttrs = 1;
        int n = 0;
        e = cudaOccupancyMaxActiveClusters(&n, wgrad_kernel<PARTS, ACC>, &c);
        if (e != cudaSuccess) return e;
        held[device] = n < 1 ? 1 : n;
    }
    *pairs = held[device];
    return cudaSuccess;
}

template <int PARTS, bool ACC>
cudaError_t launch_product(int device, const CUtensorMap& xmap, const CUtensorMap& ymap, const WgradParams& p, cudaStream_t s) {
    int pairs = 0;
    const cudaError_t e = resident_pairs<PARTS, ACC>(device, &pairs);
    if (e != cudaSuccess) return e;
    return launch_dependent(wgrad_kernel<PARTS, ACC>, 2 * (p.items < pairs ? p.items : pairs), kThreads, StageOf<PARTS>::kSmem, s, xmap,
                            ymap, p);
}

constexpr int64_t kMost = (int64_t(1) << 31) - 1024;
bool sizes_in_range(int64_t ntok, int64_t rows, int64_t dim) {
    return ntok > 0 && rows > 0 && dim > 0 && ntok <= kMost && rows <= kMost && dim <= kMost;
}

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" uint64_t lc_weight_grad_workspace(int64_t ntok, int64_t rows, int64_t dim, int32_t dy_dtype) {
    if (!sizes_in_range(ntok, rows, dim) || !elem_size(dy_dtype)) return 0;
    return uint64_t(staged_bytes(ntok, rows, dy_dtype)) + uint64_t(part_bytes(shape_of(ntok, rows, dim, dy_dtype), rows, dim));
}

extern "C" uint64_t lc_weight_grad_workspace_of(const lc_rows* dy, int64_t ntok, int64_t rows, int64_t dim) {
    if (!dy || !sizes_in_range(ntok, rows, dim) || !elem_size(dy->dtype)) return 0;
    return uint64_t(staged_dy(dy, rows) ? staged_bytes(ntok, rows, dy->dtype) : 0) +
           uint64_t(part_bytes(shape_of(ntok, rows, dim, dy->dtype), rows, dim));
}

extern "C" lc_status lc_weight_grad(int device, void* cuda_stream, const lc_rows* dy, const lc_act* x, int64_t ntok,
                                    int64_t rows, int64_t dim, const lc_rows* dw, int32_t accumulate, void* workspace,
                                    uint64_t workspace_bytes) {
    const char* call = "lc_weight_grad";
    set_last_error("");
    if (ntok < 0 || rows <= 0 || dim <= 0 || ntok > kMost / 3 || rows > kMost || dim > kMost)
        return fail_status(LC_ERR_INVALID_ARG, "%s: %lld tokens, %lld rows of %lld", call, (long long)ntok,
                           (long long)rows, (long long)dim);
    lc_status st = ops_check_rows(call, "dy", dy, ntok, rows, false);
    if (st == LC_OK) st = ops_check_act(call, x, ntok, dim);
    if (st == LC_OK) st = ops_check_rows(call, "dw", dw, rows, dim, true);
    if (st != LC_OK) return st;
    const uint64_t need = lc_weight_grad_workspace_of(dy, ntok, rows, dim);
    if (workspace_bytes < need)
        return fail_status(LC_ERR_CAPACITY, "%s: %llu bytes of workspace, %llu needed", call,
                           (unsigned long long)workspace_bytes, (unsigned long long)need);
    if (need && reinterpret_cast<uintptr_t>(workspace) % 256)
        return fail_status(LC_ERR_INVALID_ARG, "%s: the workspace is not 256-byte aligned", call);
    OnDevice cur(device);
    const int64_t blocks = (dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    const Span2 spans[] = {span_of("dy", dy, ntok, rows, false),
                           {"q", x->q, ntok, blocks * LC_ACT_BLOCK, x->q_stride, false},
                           {"e", x->e, ntok, blocks, x->e_stride, false},
                           span_of("dw", dw, rows, dim, true),
                           {"workspace", workspace, 1, int64_t(need), 0, true}};
    st = ops_check(call, device, spans, 5);
    if (st != LC_OK) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "%s: cannot make device %d current", call, device);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const int64_t dw_pitch = dw->stride * elem_size(dw->dtype);
    cudaGetLastError();
    if (ntok == 0) {
        if (accumulate) return LC_OK;
        const int64_t width = dim * elem_size(dw->dtype);
        return ops_launched(call, rows == 1 || dw_pitch == width
                                      ? cudaMemsetAsync(dw->data, 0, size_t(width * rows), s)
                                      : cudaMemset2DAsync(dw->data, size_t(dw_pitch), 0, size_t(width), size_t(rows), s));
    }
    const Shape sh = shape_of(ntok, rows, dim, dy->dtype);
    const int64_t tiles = sh.tiles_n * sh.tiles_k;
    if (tiles * sh.splits > kMost) return fail_status(LC_ERR_INVALID_ARG, "%s: too many outputs", call);
    const int64_t dy_pitch = dy->stride * elem_size(dy->dtype);
    const bool f32 = dy->dtype == LC_F32;
    const bool staged = staged_dy(dy, rows);
    uint8_t* const stage = static_cast<uint8_t*>(workspace) + part_bytes(sh, rows, dim);
    const void* ydata = dy->data;
    int64_t ypitch = dy_pitch, yrows = ntok, ycols = rows, tok_part = 0;
    cudaError_t e = cudaSuccess;
    if (staged) {
        StageParams q{};
        q.dy = static_cast<const uint8_t*>(dy->data);
        q.out = reinterpret_cast<__nv_bfloat16*>(stage);
        q.dy_pitch = dy_pitch;
        q.tok_pad = al(ntok, kTok);
        q.col_pad = al(rows, 64);
        q.ntok = ntok;
        q.rows = rows;
        q.f32 = f32;
        const int64_t grid = (q.tok_pad * q.col_pad + 1023) / 1024;
        if (grid > kMost) return fail_status(LC_ERR_INVALID_ARG, "%s: dy is too large", call);
        wgrad_stage_kernel<<<unsigned(grid), 256, 0, s>>>(q);
        e = cudaGetLastError();
        if (e != cudaSuccess) return ops_launched(call, e);
        ydata = stage;
        ypitch = q.col_pad * 2;
        ycols = q.col_pad;
        tok_part = q.tok_pad;
        yrows = q.tok_pad * (f32 ? 3 : 1);
    }
    CUtensorMap xmap, ymap;
    if (!encode(&xmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, x->q, blocks * LC_ACT_BLOCK, ntok, x->q_stride, kHalf, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !encode(&ymap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, ydata, ycols, yrows, ypitch, kBox, CU_TENSOR_MAP_SWIZZLE_128B))
        return fail_status(LC_ERR_CUDA, "%s: no tensor map", call);
    WgradParams p{};
    p.e = x->e;
    p.dw = static_cast<uint8_t*>(dw->data);
    p.part = static_cast<float*>(workspace);
    p.e_pitch = x->e_stride;
    p.dw_pitch = dw_pitch;
    p.ntok = int32_t(ntok);
    p.rows = int32_t(rows);
    p.dim = int32_t(dim);
    p.items = int32_t(tiles * sh.splits);
    p.ntiles_n = int32_t(sh.tiles_n);
    p.stages = int32_t(sh.stages);
    p.splits = int32_t(sh.splits);
    p.per_split = int32_t(sh.per_split);
    p.tok_part = int32_t(tok_part);
    p.dw_bf16 = dw->dtype == LC_BF16;
    p.stall = ops_stall();
    const bool add = accumulate && sh.splits == 1;
    if (f32) e = add ? launch_product<3, true>(device, xmap, ymap, p, s) : launch_product<3, false>(device, xmap, ymap, p, s);
    else e = add ? launch_product<1, true>(device, xmap, ymap, p, s) : launch_product<1, false>(device, xmap, ymap, p, s);
    if (e == cudaSuccess && sh.splits > 1) {
        JoinParams j{p.part, p.dw, dw_pitch, rows, dim, p.splits, accumulate != 0, p.dw_bf16};
        e = launch_dependent(wgrad_join_kernel, int(rows * ((dim + 1023) / 1024)), 256, 0, s, j);
    }
    return ops_launched(call, e);
}
