// lc_rows.cuh -- what kernels that work row by row share (lc_norm.cu, lc_addnorm.cu):
// sums over the threads of a row, and rings of rows in shared memory that bulk
// copies fill ahead of them.
#pragma once

#include "lc_bulk.cuh"
#include "lc_ops.cuh"

namespace lc {
namespace {

// The threads of a group meet.  NT: threads of its CTA; several groups have a
// barrier each, besides the CTA's own (0) where the sixteen that there are suffice.
template <int G, int NT>
__device__ __forceinline__ void group_barrier() {
    if constexpr (G == 32) __syncwarp();
    else if constexpr (NT == G) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(int(threadIdx.x) / G + (NT / G < 16 ? 1 : 0)), "n"(G) : "memory");
}

// Sums of N values (1 or 2) over the group's G threads; every thread gets them.
// Two values share the steps of a warp: after the first, one half of it works on
// either.  `slot` alternates, so one barrier a sum is enough.
template <int G, int NT, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float (*shared)[N][32], int& slot) {
    const int lane = threadIdx.x & 31;
    float x = v[0];
    if constexpr (N == 2) {
        const bool up = lane & 16;
        x = (up ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, up ? v[0] : v[1], 16);
    } else {
        x += __shfl_xor_sync(0xffffffffu, x, 16);
    }
#pragma unroll
    for (int o = 8; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if constexpr (G == 32) {
        v[0] = N == 2 ? __shfl_sync(0xffffffffu, x, 0) : x;
        if constexpr (N == 2) v[1] = __shfl_sync(0xffffffffu, x, 16);
    } else {
        const int warp = threadIdx.x >> 5;
        if (lane == 0) shared[slot][0][warp] = x;
        if (N == 2 && lane == 16) shared[slot][N - 1][warp] = x;
        group_barrier<G, NT>();
        const int w0 = NT == G ? 0 : int(threadIdx.x) / G * (G / 32);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float* from = &shared[slot][k][w0];
            if constexpr (G > 256) {
                // more warps than a thread should add up: a lane each
                float s = lane < G / 32 ? from[lane] : 0.0f;
#pragma unroll
                for (int o = 16; o; o >>= 1)
                    if (o < G / 32) s += __shfl_xor_sync(0xffffffffu, s, o);
                v[k] = __shfl_sync(0xffffffffu, s, 0);
            } else if constexpr (G == 64) {
                const float2 s = *reinterpret_cast<const float2*>(from);
                v[k] = s.x + s.y;
            } else {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < G / 32; w += 4) {
                    const float4 q = *reinterpret_cast<const float4*>(from + w);
                    s += (q.x + q.y) + (q.z + q.w);
                }
                v[k] = s;
            }
        }
        slot ^= 1;
    }
}

// --- rows through shared memory ---------------------------------------------------

constexpr int kRingMax = 8;               // rows that a group has in flight at most
constexpr size_t kRingSmem = 224 * 1024;  // of a CTA, with the barriers and sums that are not dynamic

// A group's ring: `depth` rows of `bytes`, filled by the group's first thread.
struct RowRing {
    uint32_t data, bar;      // shared-memory addresses of this group's part
    uint32_t bytes;
    int depth, at = 0;
    uint32_t round = 0;
    __device__ __forceinline__ uint32_t row() const { return data + at * bytes; }
    __device__ __forceinline__ uint32_t full() const { return bar + at * 8; }
    __device__ __forceinline__ void next() {
        if (++at == depth) {
            at = 0;
            round ^= 1;
        }
    }
};

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// A warp's wait for its row.  After one that ran out it waits for nothing any more: the
// rows that follow become NaN, since its part of their sums is, and its group still meets
// at its barriers.  The outcome is the warp's own; a group whose first warp gave up asks
// for no more rows, and its others give up where those would be.
__device__ __forceinline__ bool ring_wait(const RowRing& ring, volatile uint32_t& lost) {
    if (lost) return false;
    if (mbar_wait_warp(ring.full(), ring.round)) return true;
    lost = 1;
    return false;
}

// After a wait that ran out: what is still on its way lands before the memory is given
// back.  The rows that were not waited for left the ring's rounds behind, so a wait for
// each parity: one of them is the round that a place is in.
__device__ __forceinline__ void ring_drain(const RowRing& ring, uint32_t lost, int t) {
    if (!lost || t) return;
    for (int i = 0; i < 2 * ring.depth; ++i) mbar_wait_bounded(ring.bar + 8 * (i >> 1), i & 1, kDrainNs);
}

// Weight or bias as fp32 in the order in which the threads of a group take them:
// [VPT * V / 4][G] of four.
template <int V, int G, int VPT>
__device__ __forceinline__ void stage_param(float4* out, const uint8_t* p, bool bf16, int dim, int threads) {
    for (int k = threadIdx.x; k < VPT * V / 4 * G; k += threads) {
        const int c = (k / G / (V / 4) * G + k % G) * V + k / G % (V / 4) * 4;
        float w[4];
#pragma unroll
        for (int m = 0; m < 4; ++m)
            w[m] = c + m >= dim ? 0.0f
                   : bf16       ? to_f32(reinterpret_cast<const __nv_bfloat16*>(p)[c + m])
                                : reinterpret_cast<const float*>(p)[c + m];
        out[k] = make_float4(w[0], w[1], w[2], w[3]);
    }
}

// Shared memory above 48 KB has to be asked for, once for a kernel and device.
template <typename K>
cudaError_t allow_smem(K kernel, bool (&ready)[kOpsMaxDevices]) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && !ready[dev]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kRingSmem));
        ready[dev] = e == cudaSuccess;
    }
    return e;
}

// Rows of a group's ring in what the parameters leave of shared memory (0: none fits).
int ring_depth(size_t params, int groups, size_t row) {
    if (params + groups * row > kRingSmem) return 0;
    const size_t n = (kRingSmem - params) / (groups * row);
    return n < kRingMax ? int(n) : kRingMax;
}

}  // namespace
}  // namespace lc
