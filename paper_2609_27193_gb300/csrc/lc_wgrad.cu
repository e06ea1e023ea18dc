// lc_wgrad.cu -- the weight gradient of a linear layer whose input was kept in 8
// bits: dw[n][k] = sum over t of dy[t][n] * q[t][k] * 2^e[t][k / 128].
//
// A matrix product over the tokens on the 5th-generation tensor cores.  A value of
// the checkpoint is exactly a bf16 number, so it is an operand without a rounding;
// it is made on the way, never stored: bulk tensor copies bring 8-bit tiles of the
// checkpoint and bf16 tiles of dy into shared memory, converter warps turn the
// 8-bit tile into bf16 and write it to tensor memory, one operand of the product;
// the other is dy's tile in shared memory as it came (its rows are tokens, so both
// operands are read along the output dimensions).  The accumulator is fp32 in
// tensor memory.
//
//   warp 0    one thread issues the copies of a stage (64 tokens)
//   warp 1    one thread issues the products of a stage
//   warps 4-11 convert a stage each (a lane is a feature, a warp 32 tokens of 32
//             features), and write the outputs at the end
//
// A 32-bit dy is split into three bf16 parts that add up to it exactly (8 + 8 + 8
// bits of significand, cut off, not rounded, so nothing overflows), and a bf16 dy
// off 16-byte boundaries is copied to aligned rows, both into the workspace by a
// kernel of their own.  Few output tiles are split over the tokens; the parts are
// added in order by another kernel.
//
// Waits are bounded: one that runs out leaves NaN in the tile's outputs.
#include <cuda.h>

#include "lc_bulk.cuh"
#include "lc_ops.cuh"

namespace lc {
namespace {

constexpr int kTileK = 128;      // features of a tile: the lanes of tensor memory, and one exponent a token
constexpr int kTileN = 256;      // columns of dy of a tile
constexpr int kTok = 64;         // tokens of a stage
constexpr int kStages = 5;
constexpr int kXBytes = kTok * kTileK;             // 8-bit tile
constexpr int kBox = 64;                           // columns of one dy copy: 128 bytes, the swizzle's span
constexpr int kBoxBytes = kTok * kBox * 2;
constexpr int kYBytes = kTileN / kBox * kBoxBytes;
constexpr int kStageBytes = kXBytes + kYBytes;
constexpr int kConvWarp = 4, kConvWarps = 8;       // first converter warp (a multiple of 4), their number
constexpr int kThreads = (kConvWarp + kConvWarps) * 32;
constexpr int kTmemCols = 512;
constexpr int kAcol = kTileN;                      // tensor memory: accumulator, then a stage's operand each
constexpr int kAcols = kTok / 2;
static_assert(kAcol + kStages * kAcols <= kTmemCols, "tensor memory");
constexpr int kSmem = kStages * kStageBytes + 1024;   // and room to align the tiles to 1024 bytes

// Instruction descriptor: fp32 accumulator, bf16 operands, the first from tensor
// memory, the second with its rows along the reduction; 128 x 256.
constexpr uint32_t kIdesc = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 16 | uint32_t(kTileN / 8) << 17 | uint32_t(kTileK / 16) << 24;

struct WgradParams {
    const int8_t* e;
    uint8_t* dw;
    float* part;           // [splits][rows][dim] (splits > 1)
    int64_t e_pitch, dw_pitch;
    int32_t ntok, rows, dim;
    int32_t ntiles_n, stages, stages_part, parts, splits, per_split;   // stages of a dy part, of all parts, of a split
    int32_t tok_part;      // rows of dy between the parts
    int32_t accumulate, dw_bf16;
};

__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// d += a * b: a in tensor memory, b in shared memory.
__device__ __forceinline__ void tc_mma(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(add)
        : "memory");
}

// Shared-memory descriptor of a dy tile: 64-column boxes of 128-byte swizzled
// rows, 8 tokens 1024 bytes apart, the next 64 columns a box further.
__device__ __forceinline__ uint64_t y_desc(uint32_t addr) {
    return uint64_t((addr & 0x3ffffu) >> 4) | uint64_t(kBoxBytes >> 4) << 16 | uint64_t(1024 >> 4) << 32 |
           uint64_t(1) << 46 | uint64_t(2) << 61;
}

__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
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

// Two values of the checkpoint (bytes 0 and 2 of `q`) as bf16, times their tokens'
// scales.  A byte's low seven bits go into the fraction of 128; 128, or 256 for a
// negative one, comes off again: exact, as is the product with a power of two.
__device__ __forceinline__ uint32_t act_pair(uint32_t q, uint32_t scale) {
    const uint32_t v = (q & 0x007f007fu) | 0x43004300u, c = (q & 0x00800080u) | 0x43004300u;
    __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&c));
    d = __hmul2(d, *reinterpret_cast<const __nv_bfloat162*>(&scale));
    return *reinterpret_cast<const uint32_t*>(&d);
}

__global__ void __launch_bounds__(kThreads, 1)
    wgrad_kernel(const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CUtensorMap ymap, WgradParams p) {
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t bars[3 * kStages + 1];   // full, converted, empty; all products done
    __shared__ uint32_t tmem_base;
    __shared__ volatile uint32_t failed;
    __shared__ __align__(16) uint16_t scales[kConvWarps][2][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t tiles = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t full = smem_addr(bars), conv = full + 8 * kStages, empty = conv + 8 * kStages, done = empty + 8 * kStages;
    const int tile = blockIdx.x / p.splits, split = blockIdx.x % p.splits;
    const int n0 = tile % p.ntiles_n * kTileN, k0 = tile / p.ntiles_n * kTileK;
    const int s0 = split * p.per_split, s1 = s0 + p.per_split < p.stages ? s0 + p.per_split : p.stages;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(conv + 8 * i, kConvWarps);
            mbar_init(empty + 8 * i, 1);
        }
        mbar_init(done, 1);
        failed = 0;
        mbar_init_fence();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    dependency_wait();

    if (warp == 0) {
        if (lane == 0) {
            int s = s0;
            for (; s < s1; ++s) {
                const int i = s - s0, b = i % kStages;
                if (i >= kStages && !mbar_wait_bounded(empty + 8 * b, (i / kStages - 1) & 1, kWaitNs)) {
                    failed = 1;
                    break;
                }
                const int part = s / p.stages_part, t = (s - part * p.stages_part) * kTok;
                const uint32_t at = tiles + b * kStageBytes;
                mbar_expect_tx(full + 8 * b, kStageBytes);
                tma_2d(at + kYBytes, &xmap, k0, t, full + 8 * b);
                for (int j = 0; j < kTileN / kBox; ++j)
                    tma_2d(at + j * kBoxBytes, &ymap, n0 + j * kBox, part * p.tok_part + t, full + 8 * b);
            }
            // every copy lands before the CTA's memory is given back
            for (int i = s - s0 > kStages ? s - s0 - kStages : 0; i < s - s0; ++i)
                if (!mbar_wait_bounded(full + 8 * (i % kStages), (i / kStages) & 1, kWaitNs)) failed = 1;
        }
    } else if (warp == 1) {
        if (lane == 0) {
            bool ok = true;
            for (int s = s0; s < s1 && ok; ++s) {
                const int i = s - s0, b = i % kStages;
                ok = mbar_wait_bounded(full + 8 * b, (i / kStages) & 1, kWaitNs) &&
                     mbar_wait_bounded(conv + 8 * b, (i / kStages) & 1, kWaitNs);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t y = tiles + b * kStageBytes, a = tmem + kAcol + b * kAcols;
#pragma unroll
                for (int k = 0; k < kTok / 16; ++k) tc_mma(tmem, a + k * 8, y_desc(y + k * 2048), kIdesc, i > 0 || k > 0);
                tc_commit(empty + 8 * b);
            }
            if (!ok) failed = 1;
            tc_commit(done);
            if (!ok) mbar_wait_bounded(done, 0, kDrainNs);   // what was issued ends before the memory is given back
        }
    } else if (warp >= kConvWarp) {
        const int w = warp - kConvWarp, quad = warp & 3, half = w >> 2;
        const int t_in = half * 32;
        const int8_t* ep = p.e + k0 / LC_ACT_BLOCK;
        auto exponent = [&](int s) -> int {
            const int t = s % p.stages_part * kTok + t_in + lane;
            return s < s1 && t < p.ntok ? int(__ldg(ep + int64_t(t) * p.e_pitch)) : 0;
        };
        bool ok = true;
        int e_next = exponent(s0);
        for (int s = s0; s < s1; ++s) {
            const int i = s - s0, b = i % kStages;
            const int e = e_next;
            e_next = exponent(s + 1);
            // 2^e as bf16 (the upper half of the fp32 number), NaN for 127
            scales[w][i & 1][lane] = e == 127 ? uint16_t(0x7fff) : uint16_t((e + 127) << 7);
            __syncwarp();
            if (!mbar_wait_warp(full + 8 * b, (i / kStages) & 1)) {
                ok = false;
                break;
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint8_t* x = raw + (tiles - smem_addr(raw)) + b * kStageBytes + kYBytes + t_in * kTileK + quad * 32 + lane;
            uint32_t a[16];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint4 sc = *reinterpret_cast<const uint4*>(&scales[w][i & 1][8 * k]);
                const uint32_t s2[4] = {sc.x, sc.y, sc.z, sc.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int t = 8 * k + 2 * j;
                    a[4 * k + j] = act_pair(__byte_perm(x[t * kTileK], x[(t + 1) * kTileK], 0x5410), s2[j]);
                }
            }
            tmem_st16(tmem + (uint32_t(quad * 32) << 16) + kAcol + b * kAcols + t_in / 2, a);
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            mbar_arrive_warp(conv + 8 * b, lane);
        }
        if (ok) ok = mbar_wait_warp(done, 0);
        if (!ok) failed = 1;
        __syncwarp();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const bool bad = failed != 0;
        const int k = k0 + quad * 32 + lane;
        for (int c = 0; c < kTileN / 2; c += 16) {
            const int nc = half * (kTileN / 2) + c;
            if (n0 + nc >= p.rows) break;
            uint32_t r[16];
            __syncwarp();
            tmem_ld16(tmem + (uint32_t(quad * 32) << 16) + nc, r);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int n = n0 + nc + j;
                if (n >= p.rows || k >= p.dim) continue;
                float v = bad ? __uint_as_float(0x7fffffffu) : __uint_as_float(r[j]);
                if (p.splits > 1) {
                    p.part[(int64_t(split) * p.rows + n) * p.dim + k] = v;
                } else if (p.dw_bf16) {
                    __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.dw + n * p.dw_pitch) + k;
                    *o = __float2bfloat16_rn(p.accumulate ? __bfloat162float(*o) + v : v);
                } else {
                    float* o = reinterpret_cast<float*>(p.dw + n * p.dw_pitch) + k;
                    *o = p.accumulate ? *o + v : v;
                }
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncwarp();
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
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
// 32-bit value.  Each part takes the next eight bits of the significand, cut off.
// An infinity or a NaN stays whole in the first part.
__global__ void __launch_bounds__(256) wgrad_stage_kernel(StageParams p) {
    dependents_may_start();
    const int64_t n = p.tok_pad * p.col_pad;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) {
        const int64_t t = i / p.col_pad, c = i - t * p.col_pad;
        const bool in = t < p.ntok && c < p.rows;
        if (!p.f32) {
            p.out[i] = in ? reinterpret_cast<const __nv_bfloat16*>(p.dy + t * p.dy_pitch)[c] : __float2bfloat16_rn(0.0f);
            continue;
        }
        const float x = in ? reinterpret_cast<const float*>(p.dy + t * p.dy_pitch)[c] : 0.0f;
        const bool finite = fabsf(x) <= 3.402823466e38f;
        float rest = x;
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            float part = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
            if (!finite) part = k ? 0.0f : x;
            p.out[k * n + i] = __float2bfloat16_rn(part);
            rest -= part;
        }
    }
}

struct JoinParams {
    const float* part;
    uint8_t* dw;
    int64_t dw_pitch, rows, dim;
    int32_t splits, accumulate, dw_bf16;
};

__global__ void __launch_bounds__(256) wgrad_join_kernel(JoinParams p) {
    dependency_wait();
    const int64_t n = p.rows * p.dim;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) {
        const int64_t r = i / p.dim, c = i - r * p.dim;
        float s = 0.0f;
#pragma unroll 4
        for (int k = 0; k < p.splits; ++k) s += p.part[k * n + i];
        if (p.dw_bf16) {
            __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.dw + r * p.dw_pitch) + c;
            *o = __float2bfloat16_rn(p.accumulate ? __bfloat162float(*o) + s : s);
        } else {
            float* o = reinterpret_cast<float*>(p.dw + r * p.dw_pitch) + c;
            *o = p.accumulate ? *o + s : s;
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
// the tiles alone leave multiprocessors idle (each split at least 4 stages long).
constexpr int kSms = 152;
struct Shape {
    int64_t tiles_n, tiles_k, stages_part, stages, splits, per_split;
};
Shape shape_of(int64_t ntok, int64_t rows, int64_t dim, int32_t dy_dtype) {
    Shape s;
    s.tiles_n = (rows + kTileN - 1) / kTileN;
    s.tiles_k = (dim + kTileK - 1) / kTileK;
    s.stages_part = (ntok + kTok - 1) / kTok;
    s.stages = s.stages_part * (dy_dtype == LC_F32 ? 3 : 1);
    const int64_t tiles = s.tiles_n * s.tiles_k;
    s.splits = tiles >= kSms ? 1 : kSms / tiles;
    if (s.splits > (s.stages + 3) / 4) s.splits = (s.stages + 3) / 4;
    if (s.splits < 1) s.splits = 1;
    s.per_split = (s.stages + s.splits - 1) / s.splits;
    s.splits = (s.stages + s.per_split - 1) / s.per_split;
    return s;
}
int64_t staged_bytes(int64_t ntok, int64_t rows, int32_t dy_dtype) {
    return al(al(ntok, kTok) * al(rows, 64) * 2 * (dy_dtype == LC_F32 ? 3 : 1), 256);
}
constexpr int64_t kMost = (int64_t(1) << 31) - 1024;

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" uint64_t lc_weight_grad_workspace(int64_t ntok, int64_t rows, int64_t dim, int32_t dy_dtype) {
    if (ntok <= 0 || rows <= 0 || dim <= 0 || ntok > kMost || rows > kMost || dim > kMost || !elem_size(dy_dtype)) return 0;
    const Shape s = shape_of(ntok, rows, dim, dy_dtype);
    // rows of dy off 16 bytes, or in 32 bits, are staged; the caller need not know which
    return uint64_t(staged_bytes(ntok, rows, dy_dtype)) + (s.splits > 1 ? uint64_t(al(s.splits * rows * dim * 4, 256)) : 0);
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
    const uint64_t need = lc_weight_grad_workspace(ntok, rows, dim, dy->dtype);
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
    const bool staged = f32 || !aligned16(dy->data) || dy_pitch % 16 || dy_pitch < rows * 2;
    const void* ydata = dy->data;
    int64_t ypitch = dy_pitch, yrows = ntok, ycols = rows, tok_part = 0;
    cudaError_t e = cudaSuccess;
    if (staged) {
        StageParams q{};
        q.dy = static_cast<const uint8_t*>(dy->data);
        q.out = static_cast<__nv_bfloat16*>(workspace);
        q.dy_pitch = dy_pitch;
        q.tok_pad = al(ntok, kTok);
        q.col_pad = al(rows, 64);
        q.ntok = ntok;
        q.rows = rows;
        q.f32 = f32;
        const int64_t want = (q.tok_pad * q.col_pad + 1023) / 1024, most = int64_t(ops_sm_count(device)) * 32;
        wgrad_stage_kernel<<<unsigned(want < most ? want : most), 256, 0, s>>>(q);
        e = cudaGetLastError();
        if (e != cudaSuccess) return ops_launched(call, e);
        ydata = workspace;
        ypitch = q.col_pad * 2;
        ycols = q.col_pad;
        tok_part = q.tok_pad;
        yrows = q.tok_pad * (f32 ? 3 : 1);
    }
    CUtensorMap xmap, ymap;
    if (!encode(&xmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, x->q, blocks * LC_ACT_BLOCK, ntok, x->q_stride, kTileK, CU_TENSOR_MAP_SWIZZLE_NONE) ||
        !encode(&ymap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, ydata, ycols, yrows, ypitch, kBox, CU_TENSOR_MAP_SWIZZLE_128B))
        return fail_status(LC_ERR_CUDA, "%s: no tensor map", call);
    WgradParams p{};
    p.e = x->e;
    p.dw = static_cast<uint8_t*>(dw->data);
    p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + staged_bytes(ntok, rows, dy->dtype));
    p.e_pitch = x->e_stride;
    p.dw_pitch = dw_pitch;
    p.ntok = int32_t(ntok);
    p.rows = int32_t(rows);
    p.dim = int32_t(dim);
    p.ntiles_n = int32_t(sh.tiles_n);
    p.stages = int32_t(sh.stages);
    p.stages_part = int32_t(sh.stages_part);
    p.splits = int32_t(sh.splits);
    p.per_split = int32_t(sh.per_split);
    p.tok_part = int32_t(tok_part);
    p.accumulate = accumulate != 0;
    p.dw_bf16 = dw->dtype == LC_BF16;
    static bool ready[kOpsMaxDevices];
    if (!ready[device]) {
        e = cudaFuncSetAttribute(wgrad_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return ops_launched(call, e);
        ready[device] = true;
    }
    e = launch_dependent(wgrad_kernel, int(tiles * sh.splits), kThreads, kSmem, s, xmap, ymap, p);
    if (e == cudaSuccess && sh.splits > 1) {
        JoinParams j{p.part, p.dw, dw_pitch, rows, dim, p.splits, p.accumulate, p.dw_bf16};
        const int64_t want = (rows * dim + 1023) / 1024, most = int64_t(ops_sm_count(device)) * 32;
        e = launch_dependent(wgrad_join_kernel, int(want < most ? want : most), 256, 0, s, j);
    }
    return ops_launched(call, e);
}
