// lc_addnorm.cu -- the root-mean-square norm of a residual sum, forward and backward:
//
//   s = x + residual,  rstd = 1 / sqrt(mean of s^2 + eps),  y = s rstd w
//   h = s rstd,  dx = dsum + rstd (dy w - h mean(dy w h)),  dw = sum over tokens of dy h
//
// with s and y on request also kept in 8 bits on the same pass.  Bound by memory: a
// value is read once and written once, the row stays in registers between the sum
// over it and the outputs.  x, y and dy have one type (T), the residual stream (residual, s,
// dsum, dx) one (R): both 16 or both 32 bits, or a 32-bit stream around 16-bit branches.
//
// Two forms of each.  Direct: the warps of a row take blocks of 128 columns, four neighbouring ones a
// lane, so that a checkpoint's block is a warp's; any address, stride and width.  Through rings:
// rows on 16-byte boundaries stream through shared memory by bulk copies, several ahead.
#include "lc_rows.cuh"

namespace lc {
namespace {

struct AddNormParams {
    const uint8_t* x;
    const uint8_t* r;
    const uint8_t* w;
    uint8_t* s;
    uint8_t* y;           // null: not wanted
    float* rstd;
    int8_t* sq;           // checkpoint of the sum (null: none)
    int8_t* se;
    int8_t* yq;           // checkpoint of y
    int8_t* ye;
    int64_t ntok, x_pitch, r_pitch, s_pitch, y_pitch, sq_pitch, se_pitch, yq_pitch, ye_pitch;
    float eps, inv_dim;
    int32_t dim, w_bf16, wide;
    int32_t stall;        // test switch: a ring's first copy announces 16 bytes that never come
};

struct AddNormGradParams {
    const uint8_t* dy;
    const uint8_t* dr;    // dsum
    const uint8_t* s;     // the sum, or
    const int8_t* q;      // its checkpoint
    const int8_t* e;
    const uint8_t* w;
    const float* rstd;
    uint8_t* dx;
    float* part;          // [CTAs][2][dim], the first of the two
    uint8_t* dw;          // where the only CTA's sums go straight (null: to part)
    int64_t ntok, dy_pitch, dr_pitch, s_pitch, q_pitch, e_pitch, dx_pitch;
    float inv_dim;
    int32_t dim, w_bf16, wide, g_bf16, accumulate;
    int32_t stall;
};

// --- direct -------------------------------------------------------------------------

// Four neighbouring values from column c of a row, zero beyond its end.
template <typename T>
__device__ __forceinline__ void load4(const uint8_t* row, bool wide, int c, int dim, float (&f)[4]) {
    const T* p = reinterpret_cast<const T*>(row) + c;
    if (wide && c + 4 <= dim) {
        if constexpr (sizeof(T) == 2) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            f[0] = __uint_as_float(v.x << 16);
            f[1] = __uint_as_float(v.x & 0xffff0000u);
            f[2] = __uint_as_float(v.y << 16);
            f[3] = __uint_as_float(v.y & 0xffff0000u);
        } else {
            const float4 v = *reinterpret_cast<const float4*>(p);
            f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = c + k < dim ? to_f32(p[k]) : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store4(uint8_t* row, bool wide, int c, int dim, const float (&f)[4]) {
    T* p = reinterpret_cast<T*>(row) + c;
    if (wide && c + 4 <= dim) {
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
        else *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k < dim) p[k] = from_f32<T>(f[k]);
    }
}
template <typename P>
__device__ __forceinline__ void load_weight4(const P& p, int c, float (&f)[4]) {
    if (p.w_bf16) load4<__nv_bfloat16>(p.w, p.wide, c, p.dim, f);
    else load4<float>(p.w, p.wide, c, p.dim, f);
}

// A warp's block into a checkpoint: four values a lane.
__device__ __forceinline__ void keep_block(int8_t* q, int8_t* e, int block, int lane, const float (&f)[4]) {
    float amax = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) amax = max_nan(amax, f[k]);
    const int code = act_code(block_amax<32>(amax));
    uint32_t w[1];
    act_bytes<4>(f, code, w);
    *reinterpret_cast<uint32_t*>(q + block * LC_ACT_BLOCK + lane * 4) = w[0];
    if (lane == 0) e[block] = int8_t(code);
}

constexpr int direct_threads(int W) { return W < 4 ? 128 : W * 32; }

// W warps a row, B blocks of 128 columns a warp: warp k has blocks k, k + W, ...
template <typename T, typename R, int W, int B>
__global__ void __launch_bounds__(direct_threads(W)) add_norm_kernel(AddNormParams p) {
    constexpr int NT = direct_threads(W), G = W * 32, ROWS = NT / G;
    __shared__ __align__(16) float shared[2][1][32];
    int slot = 0;
    const int lane = threadIdx.x & 31, warp = int(threadIdx.x) % G / 32;
    const int blocks = (p.dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    for (int64_t r = int64_t(blockIdx.x) * ROWS + threadIdx.x / G; r < p.ntok; r += int64_t(gridDim.x) * ROWS) {
        float f[B][4], g[B][4];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int c = (warp + i * W) * LC_ACT_BLOCK + lane * 4;
            load4<T>(p.x + r * p.x_pitch, p.wide, c, p.dim, f[i]);
            load4<R>(p.r + r * p.r_pitch, p.wide, c, p.dim, g[i]);
        }
        float v[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < B; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f[i][k] += g[i][k];
                v[0] = fmaf(f[i][k], f[i][k], v[0]);
            }
        group_sum<G, NT>(v, shared, slot);
        const float rstd = rsqrtf(v[0] * p.inv_dim + p.eps);
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int b = warp + i * W, c = b * LC_ACT_BLOCK + lane * 4;
            if (b >= blocks) break;
            store4<R>(p.s + r * p.s_pitch, p.wide, c, p.dim, f[i]);
            if (p.sq) keep_block(p.sq + r * p.sq_pitch, p.se + r * p.se_pitch, b, lane, f[i]);
            float w[4];
            load_weight4(p, c, w);
#pragma unroll
            for (int k = 0; k < 4; ++k) f[i][k] *= rstd * w[k];
            if (p.y) store4<T>(p.y + r * p.y_pitch, p.wide, c, p.dim, f[i]);
            if (p.yq) keep_block(p.yq + r * p.yq_pitch, p.ye + r * p.ye_pitch, b, lane, f[i]);
        }
        if (lane == 0 && warp == 0) p.rstd[r] = rstd;
    }
}

template <typename T, typename R, int W, int B, bool KEPT>
__global__ void __launch_bounds__(direct_threads(W)) add_norm_grad_kernel(AddNormGradParams p) {
    constexpr int NT = direct_threads(W), G = W * 32, ROWS = NT / G;
    __shared__ __align__(16) float shared[2][1][32];
    __shared__ float4 sums[ROWS > 1 ? W * B * 32 : 1];
    dependents_may_start();
    int slot = 0;
    const int lane = threadIdx.x & 31, warp = int(threadIdx.x) % G / 32, row = threadIdx.x / G;
    float dw[B][4];
#pragma unroll
    for (int i = 0; i < B; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) dw[i][k] = 0.0f;
    for (int64_t r = int64_t(blockIdx.x) * ROWS + row; r < p.ntok; r += int64_t(gridDim.x) * ROWS) {
        float a[B][4], h[B][4];
        const float rstd = p.rstd[r];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int b = warp + i * W, c = b * LC_ACT_BLOCK + lane * 4;
            load4<T>(p.dy + r * p.dy_pitch, p.wide, c, p.dim, a[i]);
            if constexpr (KEPT) {
                // (a row ends with a whole block)
                const bool in = b * LC_ACT_BLOCK < p.dim;
                const uint32_t q = in ? *reinterpret_cast<const uint32_t*>(p.q + r * p.q_pitch + c) : 0u;
                const float sc = in ? act_scale(p.e[r * p.e_pitch + b]) : 0.0f;
#pragma unroll
                for (int k = 0; k < 4; ++k) h[i][k] = c + k < p.dim ? float(int8_t(q >> 8 * k)) * sc : 0.0f;
            } else {
                load4<R>(p.s + r * p.s_pitch, p.wide, c, p.dim, h[i]);
            }
        }
        float v[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int c = (warp + i * W) * LC_ACT_BLOCK + lane * 4;
            float w[4];
            load_weight4(p, c, w);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                h[i][k] *= rstd;
                dw[i][k] = fmaf(a[i][k], h[i][k], dw[i][k]);
                a[i][k] *= w[k];
                v[0] = fmaf(a[i][k], h[i][k], v[0]);
            }
        }
        group_sum<G, NT>(v, shared, slot);
        const float m = v[0] * p.inv_dim;
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int c = (warp + i * W) * LC_ACT_BLOCK + lane * 4;
            if (c >= p.dim) break;
            float d[4];
            load4<R>(p.dr + r * p.dr_pitch, p.wide, c, p.dim, d);
#pragma unroll
            for (int k = 0; k < 4; ++k) d[k] = fmaf(rstd, fmaf(h[i][k], -m, a[i][k]), d[k]);
            store4<R>(p.dx + r * p.dx_pitch, p.wide, c, p.dim, d);
        }
    }
    // one row of sums for the CTA: its rows' groups add theirs in turn
    if constexpr (ROWS > 1) {
        for (int k = 0; k < ROWS; ++k) {
            if (row == k)
#pragma unroll
                for (int i = 0; i < B; ++i) {
                    float4& at = sums[(warp * B + i) * 32 + lane];
                    if (k) {
                        dw[i][0] += at.x;
                        dw[i][1] += at.y;
                        dw[i][2] += at.z;
                        dw[i][3] += at.w;
                    }
                    at = make_float4(dw[i][0], dw[i][1], dw[i][2], dw[i][3]);
                }
            __syncthreads();
        }
        if (row != ROWS - 1) return;
    }
    float* out = p.part + int64_t(blockIdx.x) * 2 * p.dim;
#pragma unroll
    for (int i = 0; i < B; ++i) {
        const int c = (warp + i * W) * LC_ACT_BLOCK + lane * 4;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (c + k >= p.dim) continue;
            if (!p.dw) {
                out[c + k] = dw[i][k];
            } else if (p.g_bf16) {
                __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.dw) + c + k;
                *o = __float2bfloat16_rn(p.accumulate ? __bfloat162float(*o) + dw[i][k] : dw[i][k]);
            } else {
                float* o = reinterpret_cast<float*>(p.dw) + c + k;
                *o = p.accumulate ? *o + dw[i][k] : dw[i][k];
            }
        }
    }
}

// --- through rings --------------------------------------------------------------------

// Values of a thread's vector of V at shared-memory address `at`, in pairs.
template <typename T, int V>
__device__ __forceinline__ void lds_pairs(uint32_t at, float2 (&f)[V / 2]) {
    if constexpr (V * sizeof(T) == 16) {
        unpack(lds128(at), f);
    } else {
        static_assert(V == 8 && sizeof(T) == 4, "two vectors");
        float2 h[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            unpack(lds128(at + 16 * k), h);
            f[2 * k] = h[0];
            f[2 * k + 1] = h[1];
        }
    }
}
template <typename T, int V>
__device__ __forceinline__ void stg_pairs(T* o, const float2 (&f)[V / 2]) {
    if constexpr (V * sizeof(T) == 16) {
        st_stream(o, pack(f));
    } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float2 h[2] = {f[2 * k], f[2 * k + 1]};
            st_stream(o + 4 * k, pack(h));
        }
    }
}

// A vector of V values into a checkpoint: a block lies in 128 / V neighbouring lanes.  All lanes take part.
template <int V>
__device__ __forceinline__ void keep_vec(int8_t* q, int8_t* e, int c, int dim, const float2 (&f)[V / 2]) {
    float amax = 0.0f, v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        v[k] = k & 1 ? f[k / 2].y : f[k / 2].x;
        amax = max_nan(amax, v[k]);
    }
    const int code = act_code(block_amax<LC_ACT_BLOCK / V>(amax));
    if (c >= (dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK * LC_ACT_BLOCK) return;
    uint32_t w[V / 4];
    act_bytes<V>(v, code, w);
    if constexpr (V == 8) *reinterpret_cast<uint2*>(q + c) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(q + c) = w[0];
    if (c % LC_ACT_BLOCK == 0) e[c / LC_ACT_BLOCK] = int8_t(code);
}

constexpr int kFwdThreads = 1024;

// A slot holds a row of x and one of the residual stream.
template <typename T, typename R, int G, int VPT>
__global__ void __launch_bounds__(kFwdThreads, 1) add_norm_ring_kernel(AddNormParams p, int depth) {
    constexpr int V = kVec<T>, NT = kFwdThreads, ROWS = NT / G;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float shared[2][1][32];
    __shared__ __align__(8) uint64_t bars[ROWS * kRingMax];
    __shared__ uint32_t lost_by[NT / 32];
    volatile uint32_t& lost = lost_by[threadIdx.x >> 5];
    int slot = 0;
    const int t = threadIdx.x % G, group = threadIdx.x / G;
    float4* params = reinterpret_cast<float4*>(smem);
    constexpr int kParam = VPT * V / 4 * G;
    const uint32_t x_bytes = uint32_t(p.dim) * uint32_t(sizeof(T)), r_bytes = uint32_t(p.dim) * uint32_t(sizeof(R));
    RowRing ring;
    ring.bytes = x_bytes + r_bytes;
    ring.depth = depth;
    ring.data = smem_addr(smem) + kParam * 16 + group * depth * ring.bytes;
    ring.bar = smem_addr(bars) + group * kRingMax * 8;
    if (threadIdx.x < ROWS * kRingMax) {
        mbar_init(smem_addr(bars) + 8 * threadIdx.x, 1);
        mbar_init_fence();
    }
    lost = 0;
    __syncthreads();
    const int64_t step = int64_t(gridDim.x) * ROWS;
    int64_t r = int64_t(group) * gridDim.x + blockIdx.x;
    int64_t ahead = r;
    auto fetch = [&](int at, uint32_t more) {
        const uint32_t to = ring.data + at * ring.bytes, bar = ring.bar + 8 * at;
        mbar_expect_tx(bar, ring.bytes + more);
        bulk_g2s(to, p.x + ahead * p.x_pitch, x_bytes, bar);
        bulk_g2s(to + x_bytes, p.r + ahead * p.r_pitch, r_bytes, bar);
    };
    if (t == 0)
        for (int i = 0; i < depth && ahead < p.ntok; ++i, ahead += step) fetch(i, i == 0 && p.stall ? 16 : 0);
    stage_param<V, G, VPT>(params, p.w, p.w_bf16, p.dim, NT);
    __syncthreads();
    for (; r < p.ntok; r += step) {
        const bool ok = ring_wait(ring, lost);
        float2 f[VPT][V / 2];
        R* s = reinterpret_cast<R*>(p.s + r * p.s_pitch);
        float2 part[2] = {both(0.0f), both(0.0f)};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (i * G + t) * V;
            if (c < p.dim) {
                float2 g[V / 2];
                lds_pairs<T, V>(ring.row() + c * int(sizeof(T)), f[i]);
                lds_pairs<R, V>(ring.row() + x_bytes + c * int(sizeof(R)), g);
#pragma unroll
                for (int k = 0; k < V / 2; ++k) {
                    f[i][k] = add2(f[i][k], g[k]);
                    part[k & 1] = fma2(f[i][k], f[i][k], part[k & 1]);
                }
                if (!ok) f[i][0].x = part[0].x = __uint_as_float(0x7fffffffu);
            } else {
#pragma unroll
                for (int k = 0; k < V / 2; ++k) f[i][k] = both(0.0f);
            }
        }
        part[0] = add2(part[0], part[1]);
        float v[1] = {part[0].x + part[0].y};
        group_sum<G, NT>(v, shared, slot);
        if (t == 0 && ahead < p.ntok && !lost) fetch(ring.at, 0);
        ahead += step;
        ring.next();
        const float rstd = rsqrtf(v[0] * p.inv_dim + p.eps);
        if (!ok) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int k = 0; k < V / 2; ++k) f[i][k] = both(__uint_as_float(0x7fffffffu));
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            if ((i * G + t) * V < p.dim) stg_pairs<R, V>(s + (i * G + t) * V, f[i]);
        if (p.sq) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) keep_vec<V>(p.sq + r * p.sq_pitch, p.se + r * p.se_pitch, (i * G + t) * V, p.dim, f[i]);
        }
        T* y = reinterpret_cast<T*>(p.y + r * p.y_pitch);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (i * G + t) * V;
#pragma unroll
            for (int k = 0; k < V / 2; k += 2) {
                const float4 w = params[(i * (V / 4) + k / 2) * G + t];
                f[i][k] = mul2(f[i][k], mul2(both(rstd), make_float2(w.x, w.y)));
                f[i][k + 1] = mul2(f[i][k + 1], mul2(both(rstd), make_float2(w.z, w.w)));
            }
            if (p.y && c < p.dim) stg_pairs<T, V>(y + c, f[i]);
        }
        if (p.yq) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) keep_vec<V>(p.yq + r * p.yq_pitch, p.ye + r * p.ye_pitch, (i * G + t) * V, p.dim, f[i]);
        }
        if (t == 0) p.rstd[r] = rstd;
    }
    ring_drain(ring, lost, t);
}

constexpr int kBwdThreads = 512;

// A slot holds the rows of dy, of dsum and of the sum (or its 8-bit values; their exponents are asked for a
// row ahead into registers).  dsum is read after the row's sum, so a slot is filled again once the threads have
// met in the next row's.
template <typename T, typename R, int G, int VPT, bool KEPT>
__global__ void __launch_bounds__(kBwdThreads, 1) add_norm_grad_ring_kernel(AddNormGradParams p, int depth) {
    constexpr int V = kVec<T>, NT = kBwdThreads, ROWS = NT / G;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float shared[2][1][32];
    __shared__ __align__(8) uint64_t bars[ROWS * kRingMax];
    __shared__ uint32_t lost_by[NT / 32];
    volatile uint32_t& lost = lost_by[threadIdx.x >> 5];
    dependents_may_start();
    int slot = 0;
    const int t = threadIdx.x % G, group = threadIdx.x / G;
    float4* params = reinterpret_cast<float4*>(smem);
    constexpr int kParam = VPT * V / 4 * G;
    const uint32_t dy_bytes = uint32_t(p.dim) * uint32_t(sizeof(T)), dr_bytes = uint32_t(p.dim) * uint32_t(sizeof(R));
    const uint32_t s_bytes = KEPT ? uint32_t(p.dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK * LC_ACT_BLOCK : dr_bytes;
    RowRing ring;
    ring.bytes = dy_bytes + dr_bytes + s_bytes;
    ring.depth = depth;
    ring.data = smem_addr(smem) + kParam * 16 + group * depth * ring.bytes;
    ring.bar = smem_addr(bars) + group * kRingMax * 8;
    if (threadIdx.x < ROWS * kRingMax) {
        mbar_init(smem_addr(bars) + 8 * threadIdx.x, 1);
        mbar_init_fence();
    }
    lost = 0;
    __syncthreads();
    const int64_t step = int64_t(gridDim.x) * ROWS;
    int64_t r = int64_t(group) * gridDim.x + blockIdx.x;
    int64_t ahead = r;
    auto fetch = [&](int at, uint32_t more) {
        const uint32_t to = ring.data + at * ring.bytes, bar = ring.bar + 8 * at;
        mbar_expect_tx(bar, ring.bytes + more);
        bulk_g2s(to, p.dy + ahead * p.dy_pitch, dy_bytes, bar);
        bulk_g2s(to + dy_bytes, p.dr + ahead * p.dr_pitch, dr_bytes, bar);
        bulk_g2s(to + dy_bytes + dr_bytes, KEPT ? reinterpret_cast<const uint8_t*>(p.q) + ahead * p.q_pitch : p.s + ahead * p.s_pitch,
                 s_bytes, bar);
    };
    if (t == 0)
        for (int i = 0; i < depth && ahead < p.ntok; ++i, ahead += step) fetch(i, i == 0 && p.stall ? 16 : 0);
    stage_param<V, G, VPT>(params, p.w, p.w_bf16, p.dim, NT);
    __syncthreads();
    float2 dw[VPT][V / 2];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V / 2; ++j) dw[i][j] = both(0.0f);
    int code[VPT];
    float rstd = 0.0f;
    auto row_values = [&](int64_t at) {   // what a row has beside its vectors
        if (at >= p.ntok) return;
        rstd = __ldg(p.rstd + at);
        if constexpr (KEPT) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int c = (i * G + t) * V;
                if (c < p.dim) code[i] = __ldg(p.e + at * p.e_pitch + c / LC_ACT_BLOCK);
            }
        }
    };
    row_values(r);
    int before = -1;             // the last row's place
    for (; r < p.ntok; r += step) {
        const bool ok = ring_wait(ring, lost);
        float2 a[VPT][V / 2], h[VPT][V / 2];   // dy, then dy w; the sum, then its normalised value
        const float rs = ok ? rstd : __uint_as_float(0x7fffffffu);
        float2 s1[2] = {both(0.0f), both(0.0f)};   // short chains
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (i * G + t) * V;
            if (c >= p.dim) break;
            lds_pairs<T, V>(ring.row() + c * int(sizeof(T)), a[i]);
            const uint32_t at = ring.row() + dy_bytes + dr_bytes + c * int(KEPT ? 1 : sizeof(R));
            if constexpr (KEPT) {
                uint32_t q[V / 4];
                if constexpr (V == 8) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(q[0]), "=r"(q[1]) : "r"(at) : "memory");
                else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(q[0]) : "r"(at) : "memory");
                // a byte + 128 in the fraction of 2^23 gives its value; the product with the scale is exact
                const float sc = act_scale(code[i]) * rs;
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    const uint32_t w = q[j / 2] ^ 0x80808080u;
                    const int b = j & 1 ? 2 : 0;
                    const float2 u = make_float2(__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7650 | b)),
                                                 __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7651 | b)));
                    h[i][j] = mul2(add2(u, both(-8388736.0f)), both(sc));
                }
            } else {
                lds_pairs<R, V>(at, h[i]);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) h[i][j] = mul2(h[i][j], both(rs));
            }
        }
        row_values(r + step);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if ((i * G + t) * V >= p.dim) break;
#pragma unroll
            for (int j = 0; j < V / 2; j += 2) {
                const float4 w4 = params[(i * (V / 4) + j / 2) * G + t];
                const float2 w[2] = {make_float2(w4.x, w4.y), make_float2(w4.z, w4.w)};
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    dw[i][j + m] = fma2(a[i][j + m], h[i][j + m], dw[i][j + m]);
                    a[i][j + m] = mul2(a[i][j + m], w[m]);
                    s1[m] = fma2(a[i][j + m], h[i][j + m], s1[m]);
                }
            }
        }
        s1[0] = add2(s1[0], s1[1]);
        float v[1] = {s1[0].x + s1[0].y};
        group_sum<G, NT>(v, shared, slot);
        if constexpr (G == 32) __syncwarp();
        if (before >= 0) {
            if (t == 0 && ahead < p.ntok && !lost) fetch(before, 0);
            ahead += step;
        }
        before = ring.at;
        const float m = v[0] * p.inv_dim * rs;
        R* dx = reinterpret_cast<R*>(p.dx + r * p.dx_pitch);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (i * G + t) * V;
            if (c >= p.dim) break;
            float2 d[V / 2];
            lds_pairs<R, V>(ring.row() + dy_bytes + c * int(sizeof(R)), d);
#pragma unroll
            for (int j = 0; j < V / 2; ++j) d[j] = fma2(h[i][j], both(-m), fma2(a[i][j], both(rs), d[j]));
            stg_pairs<R, V>(dx + c, d);
        }
        ring.next();
    }
    ring_drain(ring, lost, t);
    // one row of sums for the CTA: every group leaves its own in the rings' memory (all rows were read), and each
    // column is added over the groups in order
    if (lost) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < V / 2; ++j) dw[i][j] = both(__uint_as_float(0x7fffffffu));
    }
    float* out = p.part + int64_t(blockIdx.x) * 2 * p.dim;
    auto quad = [](const float2& x, const float2& y) { return make_float4(x.x, x.y, y.x, y.y); };
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (i * G + t) * V;
            if (c >= p.dim) break;
#pragma unroll
            for (int j = 0; j < V / 2; j += 2) *reinterpret_cast<float4*>(out + c + 2 * j) = quad(dw[i][j], dw[i][j + 1]);
        }
    } else {
        __syncthreads();
        constexpr int kQuads = VPT * V / 4 * G;
        float4* sums = reinterpret_cast<float4*>(smem);   // [groups][VPT * V / 4][G]
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < V / 2; j += 2)
                sums[group * kQuads + (i * (V / 4) + j / 2) * G + t] = quad(dw[i][j], dw[i][j + 1]);
        __syncthreads();
        for (int k = threadIdx.x; k < kQuads; k += NT) {
            const int c = (k / G / (V / 4) * G + k % G) * V + k / G % (V / 4) * 4;
            if (c >= p.dim) continue;
            float4 v = sums[k];
#pragma unroll 4
            for (int g = 1; g < ROWS; ++g) {
                const float4 x = sums[g * kQuads + k];
                v.x += x.x;
                v.y += x.y;
                v.z += x.z;
                v.w += x.w;
            }
            *reinterpret_cast<float4*>(out + c) = v;
        }
    }
}

// --- host -------------------------------------------------------------------------

template <typename T, typename R, int W, int B>
cudaError_t launch_direct(const AddNormParams& p, int sms, cudaStream_t s) {
    constexpr int NT = direct_threads(W), ROWS = NT / (W * 32);
    if (p.dim > W * B * LC_ACT_BLOCK) return cudaErrorInvalidValue;   // every column has a lane
    const int64_t want = (p.ntok + ROWS - 1) / ROWS, most = int64_t(sms) * 1024;
    cudaGetLastError();
    add_norm_kernel<T, R, W, B><<<unsigned(want < most ? want : most), NT, 0, s>>>(p);
    return cudaGetLastError();
}
template <typename T, typename R>
cudaError_t direct(const AddNormParams& p, int sms, cudaStream_t s) {
    if (p.dim <= 128) return launch_direct<T, R, 1, 1>(p, sms, s);
    if (p.dim <= 256) return launch_direct<T, R, 1, 2>(p, sms, s);
    if (p.dim <= 512) return launch_direct<T, R, 2, 2>(p, sms, s);
    if (p.dim <= 1024) return launch_direct<T, R, 4, 2>(p, sms, s);
    if (p.dim <= 2048) return launch_direct<T, R, 8, 2>(p, sms, s);
    if (p.dim <= 4096) return launch_direct<T, R, 8, 4>(p, sms, s);
    if (p.dim <= 8192) return launch_direct<T, R, 16, 4>(p, sms, s);
    return launch_direct<T, R, 16, 8>(p, sms, s);
}

template <typename T, typename R, int W, int B, bool KEPT>
cudaError_t launch_direct_grad(const AddNormGradParams& p, int sms, cudaStream_t s, int* ctas) {
    constexpr int NT = direct_threads(W), ROWS = NT / (W * 32);
    if (p.dim > W * B * LC_ACT_BLOCK) return cudaErrorInvalidValue;
    // what a multiprocessor holds at 128 registers a thread
    const int64_t want = (p.ntok + ROWS - 1) / ROWS;
    int64_t grid = int64_t(sms) * (512 / NT < 4 ? 512 / NT : 4);
    grid = grid < kGradCtas ? grid : kGradCtas;
    grid = grid < want ? grid : want;
    if (p.dw) grid = 1;
    *ctas = int(grid);
    cudaGetLastError();
    add_norm_grad_kernel<T, R, W, B, KEPT><<<unsigned(grid), NT, 0, s>>>(p);
    return cudaGetLastError();
}
template <typename T, typename R, bool KEPT>
cudaError_t direct_grad(const AddNormGradParams& p, int sms, cudaStream_t s, int* ctas) {
    if (p.dim <= 128) return launch_direct_grad<T, R, 1, 1, KEPT>(p, sms, s, ctas);
    if (p.dim <= 256) return launch_direct_grad<T, R, 1, 2, KEPT>(p, sms, s, ctas);
    if (p.dim <= 512) return launch_direct_grad<T, R, 2, 2, KEPT>(p, sms, s, ctas);
    if (p.dim <= 1024) return launch_direct_grad<T, R, 4, 2, KEPT>(p, sms, s, ctas);
    if (p.dim <= 2048) return launch_direct_grad<T, R, 8, 2, KEPT>(p, sms, s, ctas);
    if (p.dim <= 4096) return launch_direct_grad<T, R, 8, 4, KEPT>(p, sms, s, ctas);
    if (p.dim <= 8192) return launch_direct_grad<T, R, 16, 4, KEPT>(p, sms, s, ctas);
    return launch_direct_grad<T, R, 16, 8, KEPT>(p, sms, s, ctas);
}

template <typename T, typename R, int G, int VPT>
cudaError_t launch_ring(const AddNormParams& p, int sms, cudaStream_t s, bool* done) {
    constexpr int V = kVec<T>, NT = kFwdThreads, ROWS = NT / G;
    if (p.dim > G * VPT * V) return cudaErrorInvalidValue;
    static bool ready[kOpsMaxDevices];
    const size_t params = size_t(VPT) * V * G * 4, row = size_t(p.dim) * (sizeof(T) + sizeof(R));
    const int depth = ring_depth(params, ROWS, row);
    *done = depth > 0;
    if (!depth) return cudaSuccess;
    const cudaError_t e = allow_smem(add_norm_ring_kernel<T, R, G, VPT>, ready);
    if (e != cudaSuccess) return e;
    const int64_t grid = p.ntok < sms ? p.ntok : sms;
    cudaGetLastError();
    add_norm_ring_kernel<T, R, G, VPT><<<unsigned(grid), NT, params + ROWS * depth * row, s>>>(p, depth);
    return cudaGetLastError();
}
template <typename T, typename R>
cudaError_t ring(const AddNormParams& p, int sms, cudaStream_t s, bool* done) {
    constexpr int M = 8 / kVec<T>;          // 16 values a thread, from a warp a row on
    const int nv = (p.dim / kVec<T> + M - 1) / M;
    if (nv <= 32) return launch_ring<T, R, 32, M>(p, sms, s, done);
    if (nv <= 64) return launch_ring<T, R, 32, 2 * M>(p, sms, s, done);
    if (nv <= 128) return launch_ring<T, R, 64, 2 * M>(p, sms, s, done);
    if (nv <= 256) return launch_ring<T, R, 128, 2 * M>(p, sms, s, done);
    if (nv <= 512) return launch_ring<T, R, 256, 2 * M>(p, sms, s, done);
    if (nv <= 1024) return launch_ring<T, R, 512, 2 * M>(p, sms, s, done);
    return launch_ring<T, R, 1024, 2 * M>(p, sms, s, done);
}

template <typename T, typename R, int G, int VPT, bool KEPT>
cudaError_t launch_grad_ring(const AddNormGradParams& p, int sms, cudaStream_t s, int* ctas) {
    constexpr int V = kVec<T>, NT = kBwdThreads, ROWS = NT / G;
    if (p.dim > G * VPT * V) return cudaErrorInvalidValue;
    static bool ready[kOpsMaxDevices];
    const size_t params = size_t(VPT) * V * G * 4;
    const size_t row = size_t(p.dim) * (sizeof(T) + sizeof(R)) +
                       (KEPT ? (size_t(p.dim) + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK * LC_ACT_BLOCK : size_t(p.dim) * sizeof(R));
    const int depth = ring_depth(params, ROWS, row);
    *ctas = 0;
    if (depth < 2) return cudaSuccess;      // one row is filled again while the next is worked on
    const cudaError_t e = allow_smem(add_norm_grad_ring_kernel<T, R, G, VPT, KEPT>, ready);
    if (e != cudaSuccess) return e;
    int64_t grid = p.ntok < sms ? p.ntok : sms;
    grid = grid < kGradCtas ? grid : kGradCtas;
    *ctas = int(grid);
    size_t smem = params + ROWS * depth * row;
    if (ROWS > 1 && smem < ROWS * params) smem = ROWS * params;   // the groups' sums
    cudaGetLastError();
    add_norm_grad_ring_kernel<T, R, G, VPT, KEPT><<<unsigned(grid), NT, smem, s>>>(p, depth);
    return cudaGetLastError();
}
template <typename T, typename R, bool KEPT>
cudaError_t grad_ring(const AddNormGradParams& p, int sms, cudaStream_t s, int* ctas) {
    constexpr int M = 8 / kVec<T>;
    const int nv = (p.dim / kVec<T> + M - 1) / M;
    if (nv <= 32) return launch_grad_ring<T, R, 32, M, KEPT>(p, sms, s, ctas);
    if (nv <= 64) return launch_grad_ring<T, R, 32, 2 * M, KEPT>(p, sms, s, ctas);
    if (nv <= 128) return launch_grad_ring<T, R, 64, 2 * M, KEPT>(p, sms, s, ctas);
    if (nv <= 256) return launch_grad_ring<T, R, 128, 2 * M, KEPT>(p, sms, s, ctas);
    if (nv <= 512) return launch_grad_ring<T, R, 256, 2 * M, KEPT>(p, sms, s, ctas);
    if (nv <= 1024) return launch_grad_ring<T, R, 512, 2 * M, KEPT>(p, sms, s, ctas);
    return launch_grad_ring<T, R, 512, 4 * M, KEPT>(p, sms, s, ctas);
}

// Whether the rings pay (microseconds through them and directly):
//   forward    bf16: 64 rows of 768 2.4, 2.6; 2432 of 4096 10.1, 21.5; 4096 of 256 3.1, 3.2.  With a 32-bit stream only
//              where the arrays no longer stay in L2: 1024 of 4096 columns 9.8, 8.5; 608 of 8192 11.3, 13.2; 4096 of 2048
//              16.5, 22.4; fp32 2432 of 1024 6.5, 5.8; 4096 of 2048 16.0, 22.7 (the border is a round one: just above it, at
//              2432 of 2048 around bf16, the rings take 10.8 and the direct form would 9.9)
//   backward   bf16 152 of 2048 5.4, 5.0; 304 of 2048 5.6, 6.0; 16 of 4096 4.9, 6.1; with a 32-bit stream 608 of 1024 5.9,
//              6.5; 304 of 2048 6.1, 5.7; fp32 304 of 768 5.1, 4.9; 608 of 768 5.5, 6.3; 152 of 4096 5.8, 6.6
bool forward_ring(int64_t ntok, int64_t dim, bool stream32) { return !stream32 || ntok * dim >= 4900000; }
bool backward_ring(int64_t ntok, int64_t dim, bool stream32, int sms) { return dim >= 4096 || ntok >= (stream32 ? 4 : 2) * sms; }
// Tokens of a backward that one CTA takes: four rounds of the rows that it has at a time.
int64_t few(int64_t dim) { return dim <= 256 ? 16 : dim <= 512 ? 8 : 4; }
constexpr int64_t kMaxRows = int64_t(1) << 40;

// The types that go together: 0 both bf16, 1 a 32-bit stream around bf16 branches, 2 both fp32, -1 none.
int types_of(int32_t branch, int32_t stream) {
    if (branch == LC_BF16) return stream == LC_BF16 ? 0 : 1;
    return stream == LC_F32 ? 2 : -1;
}
bool same_array(const lc_rows* a, const lc_rows* b) { return a->data == b->data && a->stride == b->stride && a->dtype == b->dtype; }
bool wide_rows(const void* p, int64_t pitch, int64_t to) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(to) == 0 && pitch % to == 0; }

lc_status check_weight(const char* call, const void* w, int64_t dim, int32_t dtype) {
    const int e = elem_size(dtype);
    if (!w || !e || reinterpret_cast<uintptr_t>(w) % uintptr_t(e))
        return fail_status(LC_ERR_INVALID_ARG, "%s: weight is NULL, misaligned or of unknown dtype", call);
    return LC_OK;
}

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" lc_status lc_add_norm(int device, void* cuda_stream, const lc_rows* x, const lc_rows* residual, int64_t ntok,
                                 int64_t dim, const void* weight, int32_t w_dtype, double eps, const lc_rows* sum,
                                 const lc_rows* y, float* rstd, const lc_act* keep, const lc_act* y8) {
    const char* call = "lc_add_norm";
    set_last_error("");
    if (ntok < 0 || ntok > kMaxRows || dim <= 0 || dim > LC_NORM_MAX_DIM)
        return fail_status(LC_ERR_INVALID_ARG, "%s: %lld rows of %lld (at most LC_NORM_MAX_DIM = %d)", call, (long long)ntok,
                           (long long)dim, LC_NORM_MAX_DIM);
    if (!(eps >= 0.0) || eps > 1e30) return fail_status(LC_ERR_INVALID_ARG, "%s: eps %g", call, eps);
    lc_status st = ops_check_rows(call, "x", x, ntok, dim, false);
    if (st == LC_OK) st = ops_check_rows(call, "residual", residual, ntok, dim, false);
    if (st == LC_OK) st = ops_check_rows(call, "sum", sum, ntok, dim, true);
    if (st == LC_OK && y) st = ops_check_rows(call, "y", y, ntok, dim, true);
    if (st == LC_OK && keep) st = ops_check_act(call, keep, ntok, dim);
    if (st == LC_OK && y8) st = ops_check_act(call, y8, ntok, dim);
    if (st == LC_OK) st = check_weight(call, weight, dim, w_dtype);
    if (st != LC_OK) return st;
    const int types = types_of(x->dtype, residual->dtype);
    if (types < 0 || sum->dtype != residual->dtype || (y && y->dtype != x->dtype))
        return fail_status(LC_ERR_INVALID_ARG, "%s: the sum has the residual's type, y has x's, and a fp32 x goes with a fp32 residual", call);
    if (!y && !y8) return fail_status(LC_ERR_INVALID_ARG, "%s: y or its checkpoint is needed", call);
    if (reinterpret_cast<uintptr_t>(rstd) % 4) return fail_status(LC_ERR_INVALID_ARG, "%s: rstd is not element-aligned", call);
    OnDevice cur(device);
    const int64_t blocks = (dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    const bool in_place = same_array(sum, residual);
    Span2 spans[10];
    int n = 0;
    spans[n++] = span_of("x", x, ntok, dim, false);
    if (!in_place) spans[n++] = span_of("residual", residual, ntok, dim, false);
    spans[n++] = {"weight", weight, 1, dim * elem_size(w_dtype), 0, false};
    spans[n++] = span_of("sum", sum, ntok, dim, true);
    if (y) spans[n++] = span_of("y", y, ntok, dim, true);
    spans[n++] = {"rstd", rstd, 1, ntok * 4, 0, true};
    if (keep) {
        spans[n++] = {"q", keep->q, ntok, blocks * LC_ACT_BLOCK, keep->q_stride, true};
        spans[n++] = {"e", keep->e, ntok, blocks, keep->e_stride, true};
    }
    if (y8) {
        spans[n++] = {"q of y", y8->q, ntok, blocks * LC_ACT_BLOCK, y8->q_stride, true};
        spans[n++] = {"e of y", y8->e, ntok, blocks, y8->e_stride, true};
    }
    st = ops_check(call, device, spans, n);
    if (st != LC_OK) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "%s: cannot make device %d current", call, device);
    if (ntok == 0) return LC_OK;
    AddNormParams p{};
    const int te = elem_size(x->dtype), re = elem_size(residual->dtype);
    p.x = static_cast<const uint8_t*>(x->data);
    p.r = static_cast<const uint8_t*>(residual->data);
    p.w = static_cast<const uint8_t*>(weight);
    p.s = static_cast<uint8_t*>(sum->data);
    p.x_pitch = x->stride * te;
    p.r_pitch = residual->stride * re;
    p.s_pitch = sum->stride * re;
    if (y) {
        p.y = static_cast<uint8_t*>(y->data);
        p.y_pitch = y->stride * te;
    }
    p.rstd = rstd;
    if (keep) {
        p.sq = keep->q;
        p.se = keep->e;
        p.sq_pitch = keep->q_stride;
        p.se_pitch = keep->e_stride;
    }
    if (y8) {
        p.yq = y8->q;
        p.ye = y8->e;
        p.yq_pitch = y8->q_stride;
        p.ye_pitch = y8->e_stride;
    }
    p.ntok = ntok;
    p.eps = float(eps);
    p.inv_dim = float(1.0 / double(dim));
    p.dim = int32_t(dim);
    p.w_bf16 = w_dtype == LC_BF16;
    p.stall = ops_stall();
    // a single row has any stride
    const int64_t px = ntok > 1 ? p.x_pitch : 0, pr = ntok > 1 ? p.r_pitch : 0, ps = ntok > 1 ? p.s_pitch : 0, py = ntok > 1 ? p.y_pitch : 0;
    p.wide = wide_rows(p.x, px, 4 * te) && wide_rows(p.r, pr, 4 * re) && wide_rows(p.s, ps, 4 * re) && wide_rows(p.y, py, 4 * te) &&
             wide_rows(p.w, 0, 4 * elem_size(w_dtype));
    const bool vec = wide_rows(p.x, px, 16) && wide_rows(p.r, pr, 16) && wide_rows(p.s, ps, 16) && wide_rows(p.y, py, 16) && dim * te % 16 == 0;
    const int sms = ops_sm_count(device);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    using B = __nv_bfloat16;
    cudaError_t err = cudaSuccess;
    bool done = false;
    if (vec && forward_ring(ntok, dim, types > 0))
        err = types == 0 ? ring<B, B>(p, sms, s, &done) : types == 1 ? ring<B, float>(p, sms, s, &done) : ring<float, float>(p, sms, s, &done);
    if (done || err != cudaSuccess) return ops_launched(call, err);
    err = types == 0 ? direct<B, B>(p, sms, s) : types == 1 ? direct<B, float>(p, sms, s) : direct<float, float>(p, sms, s);
    return ops_launched(call, err);
}

extern "C" lc_status lc_add_norm_grad(int device, void* cuda_stream, const lc_rows* dy, const lc_rows* dsum, const lc_rows* sum,
                                      const lc_act* kept, int64_t ntok, int64_t dim, const void* weight, int32_t w_dtype,
                                      const float* rstd, const lc_rows* dx, void* dweight, int32_t g_dtype, int32_t accumulate,
                                      void* workspace, uint64_t workspace_bytes) {
    const char* call = "lc_add_norm_grad";
    set_last_error("");
    if (ntok < 0 || ntok > kMaxRows || dim <= 0 || dim > LC_NORM_MAX_DIM)
        return fail_status(LC_ERR_INVALID_ARG, "%s: %lld rows of %lld (at most LC_NORM_MAX_DIM = %d)", call, (long long)ntok,
                           (long long)dim, LC_NORM_MAX_DIM);
    if ((sum == nullptr) == (kept == nullptr))
        return fail_status(LC_ERR_INVALID_ARG, "%s: one of the sum and its checkpoint is needed", call);
    lc_status st = ops_check_rows(call, "dy", dy, ntok, dim, false);
    if (st == LC_OK) st = ops_check_rows(call, "dsum", dsum, ntok, dim, false);
    if (st == LC_OK && sum) st = ops_check_rows(call, "sum", sum, ntok, dim, false);
    if (st == LC_OK && kept) st = ops_check_act(call, kept, ntok, dim);
    if (st == LC_OK) st = ops_check_rows(call, "dx", dx, ntok, dim, true);
    if (st == LC_OK) st = check_weight(call, weight, dim, w_dtype);
    if (st != LC_OK) return st;
    const int types = types_of(dy->dtype, dsum->dtype);
    if (types < 0 || dx->dtype != dsum->dtype || (sum && sum->dtype != dsum->dtype))
        return fail_status(LC_ERR_INVALID_ARG, "%s: the sum and dx have dsum's type, and a fp32 dy goes with a fp32 dsum", call);
    const int ge = elem_size(g_dtype);
    if (!ge || !dweight || reinterpret_cast<uintptr_t>(dweight) % uintptr_t(ge))
        return fail_status(LC_ERR_INVALID_ARG, "%s: dweight is NULL, misaligned or of unknown dtype", call);
    if (reinterpret_cast<uintptr_t>(rstd) % 4) return fail_status(LC_ERR_INVALID_ARG, "%s: rstd is not element-aligned", call);
    const uint64_t need = lc_norm_grad_workspace(ntok, dim);
    if (workspace_bytes < need)
        return fail_status(LC_ERR_CAPACITY, "%s: %llu bytes of workspace, %llu needed", call, (unsigned long long)workspace_bytes,
                           (unsigned long long)need);
    if (need && reinterpret_cast<uintptr_t>(workspace) % 256)
        return fail_status(LC_ERR_INVALID_ARG, "%s: the workspace is not 256-byte aligned", call);
    OnDevice cur(device);
    const int64_t blocks = (dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    const bool in_place = same_array(dx, dsum);
    Span2 spans[10];
    int n = 0;
    spans[n++] = span_of("dy", dy, ntok, dim, false);
    if (!in_place) spans[n++] = span_of("dsum", dsum, ntok, dim, false);
    if (sum) spans[n++] = span_of("sum", sum, ntok, dim, false);
    if (kept) {
        spans[n++] = {"q", kept->q, ntok, blocks * LC_ACT_BLOCK, kept->q_stride, false};
        spans[n++] = {"e", kept->e, ntok, blocks, kept->e_stride, false};
    }
    spans[n++] = {"weight", weight, 1, dim * elem_size(w_dtype), 0, false};
    spans[n++] = {"rstd", rstd, 1, ntok * 4, 0, false};
    spans[n++] = span_of("dx", dx, ntok, dim, true);
    spans[n++] = {"dweight", dweight, 1, dim * ge, 0, true};
    if (need) spans[n++] = {"workspace", workspace, 1, int64_t(need), 0, true};
    st = ops_check(call, device, spans, n);
    if (st != LC_OK) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "%s: cannot make device %d current", call, device);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (ntok == 0) return accumulate ? LC_OK : ops_launched(call, cudaMemsetAsync(dweight, 0, size_t(dim * ge), s));
    AddNormGradParams p{};
    const int te = elem_size(dy->dtype), re = elem_size(dsum->dtype);
    p.dy = static_cast<const uint8_t*>(dy->data);
    p.dy_pitch = dy->stride * te;
    p.dr = static_cast<const uint8_t*>(dsum->data);
    p.dr_pitch = dsum->stride * re;
    if (sum) {
        p.s = static_cast<const uint8_t*>(sum->data);
        p.s_pitch = sum->stride * re;
    } else {
        p.q = kept->q;
        p.e = kept->e;
        p.q_pitch = kept->q_stride;
        p.e_pitch = kept->e_stride;
    }
    p.w = static_cast<const uint8_t*>(weight);
    p.rstd = rstd;
    p.dx = static_cast<uint8_t*>(dx->data);
    p.dx_pitch = dx->stride * re;
    p.part = static_cast<float*>(workspace);
    p.ntok = ntok;
    p.inv_dim = float(1.0 / double(dim));
    p.dim = int32_t(dim);
    p.w_bf16 = w_dtype == LC_BF16;
    p.stall = ops_stall();
    const int64_t many = ntok > 1;
    p.wide = wide_rows(p.dy, many * p.dy_pitch, 4 * te) && wide_rows(p.dr, many * p.dr_pitch, 4 * re) && wide_rows(p.s, many * p.s_pitch, 4 * re) &&
             wide_rows(p.dx, many * p.dx_pitch, 4 * re) && wide_rows(p.w, 0, 4 * elem_size(w_dtype));
    // a few tokens: one CTA for all of them, whose sums need no second kernel (4 tokens of 256: 7.2 us on the host to 4.7)
    if (ntok <= few(dim)) {
        p.dw = static_cast<uint8_t*>(dweight);
        p.g_bf16 = g_dtype == LC_BF16;
        p.accumulate = accumulate != 0;
    }
    const bool vec = !p.dw && wide_rows(p.dy, many * p.dy_pitch, 16) && wide_rows(p.dr, many * p.dr_pitch, 16) && wide_rows(p.s, many * p.s_pitch, 16) &&
                     wide_rows(p.dx, many * p.dx_pitch, 16) && dim * te % 16 == 0;
    const int sms = ops_sm_count(device);
    using B = __nv_bfloat16;
    int ctas = 0;
    cudaError_t err = cudaSuccess;
    auto go = [&](auto f) { err = f(p, sms, s, &ctas); };
    if (vec && backward_ring(ntok, dim, types > 0, sms)) {
        if (types == 0) go(sum ? grad_ring<B, B, false> : grad_ring<B, B, true>);
        else if (types == 1) go(sum ? grad_ring<B, float, false> : grad_ring<B, float, true>);
        else go(sum ? grad_ring<float, float, false> : grad_ring<float, float, true>);
    }
    if (!ctas && err == cudaSuccess) {
        if (types == 0) go(sum ? direct_grad<B, B, false> : direct_grad<B, B, true>);
        else if (types == 1) go(sum ? direct_grad<B, float, false> : direct_grad<B, float, true>);
        else go(sum ? direct_grad<float, float, false> : direct_grad<float, float, true>);
    }
    if (err == cudaSuccess && !p.dw) err = norm_fold(p.part, ctas, p.dim, dweight, nullptr, g_dtype == LC_BF16, accumulate != 0, s);
    return ops_launched(call, err);
}
