// lc_norm.cu -- layer norm and root-mean-square norm of every token's vector,
// forward and backward.
//
// Forward: a group of G threads holds a row in registers, so it is read once; the
// mean, then the mean square about it (both over registers, no cancellation), then
// the output, and on request the row's 8-bit checkpoint.  Bound by memory.
//
// Backward: a group works through rows b, b + grid, ...; a thread always has the
// same columns, so the gradients of weight and bias stay in its registers over all
// its rows.  Each CTA leaves one fp32 row of sums of them, and a second kernel adds
// those rows in order: two levels, no atomics, the same bits every time.
#include "lc_ops.cuh"

namespace lc {
namespace {

constexpr int kGradCtas = 608;    // most rows of partial sums that a call leaves

struct NormParams {
    const uint8_t* x;
    const uint8_t* w;
    const uint8_t* b;
    uint8_t* y;
    float* mean;
    float* rstd;
    int8_t* q;            // checkpoint (null: none)
    int8_t* e;
    int64_t ntok, x_pitch, y_pitch, q_pitch, e_pitch;
    float eps, inv_dim;
    int32_t dim, w_bf16, rms;
};

struct NormGradParams {
    const uint8_t* dy;
    const uint8_t* x;
    const int8_t* q;
    const int8_t* e;
    const uint8_t* w;
    const float* mean;
    const float* rstd;
    uint8_t* dx;
    float* part;          // [CTAs][2][dim]
    int64_t ntok, dy_pitch, x_pitch, q_pitch, e_pitch, dx_pitch;
    float inv_dim;
    int32_t dim, w_bf16, rms, want_params;
};

// The columns that a thread of a group of G holds: VPT vectors of V, 16 bytes each
// (VEC), or as many single elements G apart.
template <int V, int G, int VPT, bool VEC>
__device__ __forceinline__ int column(int t, int i, int j) {
    return VEC ? (i * G + t) * V + j : (i * V + j) * G + t;
}

template <typename T, int G, int VPT, bool VEC>
__device__ __forceinline__ void load_row(const uint8_t* row, int t, int dim, float (&f)[VPT][kVec<T>]) {
    constexpr int V = kVec<T>;
    const T* r = reinterpret_cast<const T*>(row);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        if (VEC && column<V, G, VPT, VEC>(t, i, 0) + V <= dim) {
            unpack(ld_stream(r + column<V, G, VPT, VEC>(t, i, 0)), f[i]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = column<V, G, VPT, VEC>(t, i, j);
                f[i][j] = c < dim ? to_f32(r[c]) : 0.0f;
            }
        }
    }
}

template <typename T, int G, int VPT, bool VEC>
__device__ __forceinline__ void store_row(uint8_t* row, int t, int dim, const float (&f)[VPT][kVec<T>]) {
    constexpr int V = kVec<T>;
    T* r = reinterpret_cast<T*>(row);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        if (VEC && column<V, G, VPT, VEC>(t, i, 0) + V <= dim) {
            st_stream(r + column<V, G, VPT, VEC>(t, i, 0), pack(f[i]));
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = column<V, G, VPT, VEC>(t, i, j);
                if (c < dim) r[c] = from_f32<T>(f[i][j]);
            }
        }
    }
}

// Weight or bias at the thread's columns.
template <int V, int G, int VPT, bool VEC>
__device__ __forceinline__ void load_param(const uint8_t* p, bool bf16, int t, int i, int dim, float (&f)[V]) {
    if (VEC && column<V, G, VPT, VEC>(t, i, 0) + V <= dim) {
        const int c = column<V, G, VPT, VEC>(t, i, 0);
        if (bf16) {
            if constexpr (V == 8) {
                unpack(__ldg(reinterpret_cast<const uint4*>(p + c * 2)), f);
            } else {
                const uint2 v = __ldg(reinterpret_cast<const uint2*>(p + c * 2));
                f[0] = __uint_as_float(v.x << 16);
                f[1] = __uint_as_float(v.x & 0xffff0000u);
                f[2] = __uint_as_float(v.y << 16);
                f[3] = __uint_as_float(v.y & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int k = 0; k < V; k += 4) {
                const float4 v = __ldg(reinterpret_cast<const float4*>(p + (c + k) * 4));
                f[k] = v.x;
                f[k + 1] = v.y;
                f[k + 2] = v.z;
                f[k + 3] = v.w;
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int c = column<V, G, VPT, VEC>(t, i, j);
        f[j] = c >= dim ? 0.0f
               : bf16   ? to_f32(reinterpret_cast<const __nv_bfloat16*>(p)[c])
                        : reinterpret_cast<const float*>(p)[c];
    }
}

// Sum over the group's G threads; every thread gets it.  `slot` alternates, so one
// barrier a sum is enough.
template <int G, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float (*shared)[32][N], int& slot) {
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    if constexpr (G > 32) {
        const int warp = threadIdx.x >> 5;
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) shared[slot][warp][k] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < G / 32; ++w) s += shared[slot][w][k];
            v[k] = s;
        }
        slot ^= 1;
    }
}

constexpr int cta_threads(int G) { return G < 128 ? 128 : G; }

template <typename T, int G, int VPT, bool VEC>
__global__ void __launch_bounds__(cta_threads(G)) norm_kernel(NormParams p) {
    constexpr int V = kVec<T>;
    constexpr int R = cta_threads(G) / G;   // rows of a CTA at a time
    __shared__ float shared[2][32][1];
    int slot = 0;
    const int t = threadIdx.x % G;
    const int64_t step = int64_t(gridDim.x) * R;
    for (int64_t r = int64_t(blockIdx.x) * R + threadIdx.x / G; r < p.ntok; r += step) {
        float f[VPT][V];
        load_row<T, G, VPT, VEC>(p.x + r * p.x_pitch, t, p.dim, f);
        if constexpr (VEC) {
            if (p.q) {
                // a block of 128 values lies in 128 / V neighbouring lanes
                constexpr int L = LC_ACT_BLOCK / V;
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    float amax = 0.0f;
#pragma unroll
                    for (int j = 0; j < V; ++j) amax = max_nan(amax, f[i][j]);
                    const int code = act_code(block_amax<L>(amax));
                    const int c = column<V, G, VPT, VEC>(t, i, 0);
                    if (c < (p.dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK * LC_ACT_BLOCK) {
                        uint32_t w[V / 4];
                        act_bytes<V>(f[i], code, w);
                        int8_t* q = p.q + r * p.q_pitch + c;
                        if constexpr (V == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
                        else *reinterpret_cast<uint32_t*>(q) = w[0];
                        if (c % LC_ACT_BLOCK == 0) p.e[r * p.e_pitch + c / LC_ACT_BLOCK] = int8_t(code);
                    }
                }
            }
        }
        float s[1] = {0.0f};
        float mean = 0.0f;
        if (!p.rms) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) s[0] += f[i][j];
            group_sum<G>(s, shared, slot);
            mean = s[0] * p.inv_dim;
            s[0] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = f[i][j] - mean;
                if (column<V, G, VPT, VEC>(t, i, j) < p.dim) s[0] += d * d;
            }
        group_sum<G>(s, shared, slot);
        const float rstd = rsqrtf(s[0] * p.inv_dim + p.eps);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float w[V], b[V];
            load_param<V, G, VPT, VEC>(p.w, p.w_bf16, t, i, p.dim, w);
            if (p.b) load_param<V, G, VPT, VEC>(p.b, p.w_bf16, t, i, p.dim, b);
#pragma unroll
            for (int j = 0; j < V; ++j) f[i][j] = (f[i][j] - mean) * rstd * w[j] + (p.b ? b[j] : 0.0f);
        }
        store_row<T, G, VPT, VEC>(p.y + r * p.y_pitch, t, p.dim, f);
        if (t == 0) {
            if (!p.rms) p.mean[r] = mean;
            p.rstd[r] = rstd;
        }
    }
}

// KEPT: x comes from its checkpoint.  SMEM: the sums for weight and bias lie in
// shared memory, a slot of its own for every thread and column (rows too wide for
// registers).
template <typename T, int G, int VPT, bool VEC, bool KEPT, bool SMEM>
__global__ void __launch_bounds__(cta_threads(G)) norm_grad_kernel(NormGradParams p) {
    constexpr int V = kVec<T>;
    constexpr int R = cta_threads(G) / G;
    extern __shared__ float2 sums[];
    __shared__ float shared[2][32][2];
    int slot = 0;
    const int t = threadIdx.x % G;
    float dw[SMEM ? 1 : VPT][V], db[SMEM ? 1 : VPT][V];
    if constexpr (SMEM) {
        for (int k = 0; k < VPT * V; ++k) sums[k * G + t] = make_float2(0.0f, 0.0f);
    } else {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) dw[i][j] = db[i][j] = 0.0f;
    }
    const int64_t step = int64_t(gridDim.x) * R;
    for (int64_t r = int64_t(blockIdx.x) * R + threadIdx.x / G; r < p.ntok; r += step) {
        float g[VPT][V], h[VPT][V];
        load_row<T, G, VPT, VEC>(p.dy + r * p.dy_pitch, t, p.dim, g);
        const float mean = p.rms ? 0.0f : p.mean[r], rstd = p.rstd[r];
        if constexpr (KEPT) {
            const int8_t* q = p.q + r * p.q_pitch;
            const int8_t* ex = p.e + r * p.e_pitch;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int c0 = column<V, G, VPT, VEC>(t, i, 0);
                if (VEC && c0 + V <= p.dim) {
                    // V values of one block
                    const float s = act_scale(ex[c0 / LC_ACT_BLOCK]);
                    uint32_t w[V / 4];
                    if constexpr (V == 8) {
                        const uint2 v = __ldg(reinterpret_cast<const uint2*>(q + c0));
                        w[0] = v.x;
                        w[1] = v.y;
                    } else {
                        w[0] = __ldg(reinterpret_cast<const uint32_t*>(q + c0));
                    }
#pragma unroll
                    for (int j = 0; j < V; ++j) h[i][j] = float(int8_t(w[j / 4] >> (8 * (j % 4)))) * s;
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const int c = column<V, G, VPT, VEC>(t, i, j);
                        h[i][j] = c < p.dim ? float(q[c]) * act_scale(ex[c / LC_ACT_BLOCK]) : 0.0f;
                    }
                }
            }
        } else {
            load_row<T, G, VPT, VEC>(p.x + r * p.x_pitch, t, p.dim, h);
        }
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float w[V];
            load_param<V, G, VPT, VEC>(p.w, p.w_bf16, t, i, p.dim, w);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                h[i][j] = (h[i][j] - mean) * rstd;   // columns beyond dim: dy = 0 there, so nothing counts
                if constexpr (SMEM) {
                    float2& a = sums[(i * V + j) * G + t];
                    a.x += g[i][j] * h[i][j];
                    a.y += g[i][j];
                } else {
                    dw[i][j] += g[i][j] * h[i][j];
                    db[i][j] += g[i][j];
                }
                g[i][j] *= w[j];
                s[0] += g[i][j];
                s[1] += g[i][j] * h[i][j];
            }
        }
        group_sum<G>(s, shared, slot);
        if (p.dx) {
            const float m1 = p.rms ? 0.0f : s[0] * p.inv_dim, m2 = s[1] * p.inv_dim;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) g[i][j] = rstd * (g[i][j] - m1 - h[i][j] * m2);
            store_row<T, G, VPT, VEC>(p.dx + r * p.dx_pitch, t, p.dim, g);
        }
    }
    dependents_may_start();
    if (!p.want_params) return;
    // one row of sums for the CTA: its groups add theirs in turn
    if constexpr (R > 1) {
        static_assert(!SMEM, "narrow rows have their sums in registers");
        for (int k = 0; k < R; ++k) {
            if (int(threadIdx.x) / G == k)
#pragma unroll
                for (int i = 0; i < VPT; ++i)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        float2& a = sums[(i * V + j) * G + t];
                        if (k == 0) a = make_float2(dw[i][j], db[i][j]);
                        else {
                            dw[i][j] += a.x;
                            db[i][j] += a.y;
                            a = make_float2(dw[i][j], db[i][j]);
                        }
                    }
            __syncthreads();
        }
        if (int(threadIdx.x) / G != R - 1) return;
    }
    float* out = p.part + int64_t(blockIdx.x) * 2 * p.dim;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = column<V, G, VPT, VEC>(t, i, j);
            if (c >= p.dim) continue;
            if constexpr (SMEM) {
                out[c] = sums[(i * V + j) * G + t].x;
                out[p.dim + c] = sums[(i * V + j) * G + t].y;
            } else {
                out[c] = dw[i][j];
                out[p.dim + c] = db[i][j];
            }
        }
}

struct FoldParams {
    const float* part;
    uint8_t* dw;
    uint8_t* db;
    int32_t rows, dim, g_bf16, accumulate;
};

// Adds the CTAs' rows of sums: 32 columns a CTA, 8 threads a column, each taking
// every 8th row, their sums added in order.
__global__ void __launch_bounds__(256) norm_fold_kernel(FoldParams p) {
    __shared__ float sums[8][32];
    dependency_wait();
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), k = threadIdx.x >> 5;
    uint8_t* out = blockIdx.y ? p.db : p.dw;
    if (!out) return;
    const float* part = p.part + (blockIdx.y ? p.dim : 0);
    float s = 0.0f;
    if (c < p.dim) {
#pragma unroll 8
        for (int r = k; r < p.rows; r += 8) s += part[int64_t(r) * 2 * p.dim + c];
    }
    sums[k][threadIdx.x & 31] = s;
    __syncthreads();
    if (k || c >= p.dim) return;
    for (int i = 1; i < 8; ++i) s += sums[i][threadIdx.x];
    if (p.g_bf16) {
        __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(out) + c;
        *o = __float2bfloat16_rn(p.accumulate ? __bfloat162float(*o) + s : s);
    } else {
        float* o = reinterpret_cast<float*>(out) + c;
        *o = p.accumulate ? *o + s : s;
    }
}

template <typename T, int G, int VPT, bool VEC>
cudaError_t launch_norm(const NormParams& p, int sms, cudaStream_t s) {
    constexpr int R = cta_threads(G) / G;
    const int64_t want = (p.ntok + R - 1) / R;
    const int64_t most = int64_t(sms) * 64;
    cudaGetLastError();
    norm_kernel<T, G, VPT, VEC><<<unsigned(want < most ? want : most), cta_threads(G), 0, s>>>(p);
    return cudaGetLastError();
}

// Threads of a row and vectors of a thread: a warp up to 4 vectors a lane, then
// groups of warps with 2 a thread.
template <typename T, bool VEC>
cudaError_t dispatch_norm(const NormParams& p, int sms, cudaStream_t s) {
    const int nv = (p.dim + kVec<T> - 1) / kVec<T>;
    if (nv <= 32) return launch_norm<T, 32, 1, VEC>(p, sms, s);
    if (nv <= 64) return launch_norm<T, 32, 2, VEC>(p, sms, s);
    if (nv <= 128) return launch_norm<T, 32, 4, VEC>(p, sms, s);
    if (nv <= 256) return launch_norm<T, 128, 2, VEC>(p, sms, s);
    if (nv <= 512) return launch_norm<T, 256, 2, VEC>(p, sms, s);
    if (nv <= 1024) return launch_norm<T, 512, 2, VEC>(p, sms, s);
    if constexpr (kVec<T> == 4)
        if (nv > 2048) return launch_norm<T, 1024, 4, VEC>(p, sms, s);
    return launch_norm<T, 1024, 2, VEC>(p, sms, s);
}

template <typename T, int G, int VPT, bool VEC, bool KEPT, bool SMEM>
cudaError_t launch_grad(const NormGradParams& p, int sms, cudaStream_t s, int* ctas) {
    constexpr int R = cta_threads(G) / G;
    constexpr size_t smem = SMEM || R > 1 ? sizeof(float2) * G * VPT * kVec<T> : 0;
    auto kernel = norm_grad_kernel<T, G, VPT, VEC, KEPT, SMEM>;
    static int resident[kOpsMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!resident[dev]) {
        if (smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
        int n = 0;
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, cta_threads(G), smem);
        if (e != cudaSuccess) return e;
        resident[dev] = n < 1 ? 1 : n;
    }
    const int64_t want = (p.ntok + R - 1) / R;
    int64_t grid = int64_t(sms) * resident[dev];
    grid = grid < kGradCtas ? grid : kGradCtas;
    grid = grid < want ? grid : want;
    *ctas = int(grid);
    cudaGetLastError();
    kernel<<<unsigned(grid), cta_threads(G), smem, s>>>(p);
    return cudaGetLastError();
}

template <typename T, bool VEC, bool KEPT>
cudaError_t dispatch_grad(const NormGradParams& p, int sms, cudaStream_t s, int* ctas) {
    const int nv = (p.dim + kVec<T> - 1) / kVec<T>;
    if (nv <= 32) return launch_grad<T, 32, 1, VEC, KEPT, false>(p, sms, s, ctas);
    if (nv <= 64) return launch_grad<T, 32, 2, VEC, KEPT, false>(p, sms, s, ctas);
    if (nv <= 128) return launch_grad<T, 128, 1, VEC, KEPT, false>(p, sms, s, ctas);
    if (nv <= 256) return launch_grad<T, 256, 1, VEC, KEPT, false>(p, sms, s, ctas);
    if (nv <= 512) return launch_grad<T, 256, 2, VEC, KEPT, false>(p, sms, s, ctas);
    if (nv <= 1024) return launch_grad<T, 512, 2, VEC, KEPT, false>(p, sms, s, ctas);
    if constexpr (kVec<T> == 4)
        if (nv > 2048) return launch_grad<T, 1024, 4, VEC, KEPT, true>(p, sms, s, ctas);
    return launch_grad<T, 1024, 2, VEC, KEPT, true>(p, sms, s, ctas);
}

constexpr int64_t kMaxRows = int64_t(1) << 40;

bool plain_params(const void* w, int64_t dim, int32_t dtype) {
    return w && elem_size(dtype) && reinterpret_cast<uintptr_t>(w) % uintptr_t(elem_size(dtype)) == 0 && dim > 0;
}

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" lc_status lc_norm(int device, void* cuda_stream, int32_t kind, const lc_rows* x, int64_t ntok, int64_t dim,
                             const void* weight, const void* bias, int32_t w_dtype, double eps, const lc_rows* y,
                             float* mean, float* rstd, const lc_act* keep) {
    const char* call = "lc_norm";
    set_last_error("");
    if (kind != LC_NORM_LAYER && kind != LC_NORM_RMS)
        return fail_status(LC_ERR_INVALID_ARG, "%s: unknown kind %d", call, int(kind));
    if (ntok < 0 || ntok > kMaxRows || dim <= 0 || dim > LC_NORM_MAX_DIM)
        return fail_status(LC_ERR_INVALID_ARG, "%s: %lld rows of %lld (at most LC_NORM_MAX_DIM = %d)", call,
                           (long long)ntok, (long long)dim, LC_NORM_MAX_DIM);
    if (!(eps >= 0.0) || eps > 1e30) return fail_status(LC_ERR_INVALID_ARG, "%s: eps %g", call, eps);
    lc_status st = ops_check_rows(call, "x", x, ntok, dim, false);
    if (st == LC_OK) st = ops_check_rows(call, "y", y, ntok, dim, true);
    if (st == LC_OK && keep) st = ops_check_act(call, keep, ntok, dim);
    if (st != LC_OK) return st;
    if (y->dtype != x->dtype) return fail_status(LC_ERR_INVALID_ARG, "%s: y has another type than x", call);
    if (!plain_params(weight, dim, w_dtype) || (bias && !plain_params(bias, dim, w_dtype)))
        return fail_status(LC_ERR_INVALID_ARG, "%s: weight or bias is NULL, misaligned or of unknown dtype", call);
    if (ntok > 0 && (kind == LC_NORM_RMS) != (mean == nullptr))
        return fail_status(LC_ERR_INVALID_ARG, "%s: mean goes with LC_NORM_LAYER, and only with it", call);
    if (reinterpret_cast<uintptr_t>(mean) % 4 || reinterpret_cast<uintptr_t>(rstd) % 4)
        return fail_status(LC_ERR_INVALID_ARG, "%s: mean or rstd is not element-aligned", call);
    OnDevice cur(device);
    const int we = elem_size(w_dtype);
    const int64_t blocks = (dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    Span2 spans[8];
    int n = 0;
    spans[n++] = span_of("x", x, ntok, dim, false);
    spans[n++] = {"weight", weight, 1, dim * we, 0, false};
    if (bias) spans[n++] = {"bias", bias, 1, dim * we, 0, false};
    spans[n++] = span_of("y", y, ntok, dim, true);
    if (mean) spans[n++] = {"mean", mean, 1, ntok * 4, 0, true};
    spans[n++] = {"rstd", rstd, 1, ntok * 4, 0, true};
    if (keep) {
        spans[n++] = {"q", keep->q, ntok, blocks * LC_ACT_BLOCK, keep->q_stride, true};
        spans[n++] = {"e", keep->e, ntok, blocks, keep->e_stride, true};
    }
    st = ops_check(call, device, spans, n);
    if (st != LC_OK) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "%s: cannot make device %d current", call, device);
    if (ntok == 0) return LC_OK;
    NormParams p{};
    p.x = static_cast<const uint8_t*>(x->data);
    p.w = static_cast<const uint8_t*>(weight);
    p.b = static_cast<const uint8_t*>(bias);
    p.y = static_cast<uint8_t*>(y->data);
    p.mean = mean;
    p.rstd = rstd;
    p.ntok = ntok;
    const int e = elem_size(x->dtype);
    p.x_pitch = x->stride * e;
    p.y_pitch = y->stride * e;
    p.eps = float(eps);
    p.inv_dim = float(1.0 / double(dim));
    p.dim = int32_t(dim);
    p.w_bf16 = w_dtype == LC_BF16;
    p.rms = kind == LC_NORM_RMS;
    const bool vec = aligned16(p.x) && aligned16(p.y) && aligned16(p.w) && aligned16(p.b) && p.x_pitch % 16 == 0 &&
                     p.y_pitch % 16 == 0;
    const int sms = ops_sm_count(device);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (keep && vec) {
        p.q = keep->q;
        p.e = keep->e;
        p.q_pitch = keep->q_stride;
        p.e_pitch = keep->e_stride;
    } else if (keep) {
        // rows off 16 bytes: a lane's columns are not one block's, so the checkpoint has a pass of its own
        const cudaError_t err = act_save_rows(x, keep, ntok, dim, s);
        if (err != cudaSuccess) return ops_launched(call, err);
    }
    cudaError_t err;
    if (x->dtype == LC_BF16)
        err = vec ? dispatch_norm<__nv_bfloat16, true>(p, sms, s) : dispatch_norm<__nv_bfloat16, false>(p, sms, s);
    else
        err = vec ? dispatch_norm<float, true>(p, sms, s) : dispatch_norm<float, false>(p, sms, s);
    return ops_launched(call, err);
}

extern "C" uint64_t lc_norm_grad_workspace(int64_t ntok, int64_t dim) {
    if (ntok <= 0 || dim <= 0 || dim > LC_NORM_MAX_DIM) return 0;
    return uint64_t(ntok < kGradCtas ? ntok : kGradCtas) * 2 * uint64_t(dim) * 4;
}

extern "C" lc_status lc_norm_grad(int device, void* cuda_stream, int32_t kind, const lc_rows* dy, const lc_rows* x,
                                  const lc_act* kept, int64_t ntok, int64_t dim, const void* weight, int32_t w_dtype,
                                  const float* mean, const float* rstd, const lc_rows* dx, void* dweight, void* dbias,
                                  int32_t g_dtype, int32_t accumulate, void* workspace, uint64_t workspace_bytes) {
    const char* call = "lc_norm_grad";
    set_last_error("");
    if (kind != LC_NORM_LAYER && kind != LC_NORM_RMS)
        return fail_status(LC_ERR_INVALID_ARG, "%s: unknown kind %d", call, int(kind));
    if (ntok < 0 || ntok > kMaxRows || dim <= 0 || dim > LC_NORM_MAX_DIM)
        return fail_status(LC_ERR_INVALID_ARG, "%s: %lld rows of %lld (at most LC_NORM_MAX_DIM = %d)", call,
                           (long long)ntok, (long long)dim, LC_NORM_MAX_DIM);
    if ((x == nullptr) == (kept == nullptr))
        return fail_status(LC_ERR_INVALID_ARG, "%s: one of x and its checkpoint is needed", call);
    lc_status st = ops_check_rows(call, "dy", dy, ntok, dim, false);
    if (st == LC_OK && x) st = ops_check_rows(call, "x", x, ntok, dim, false);
    if (st == LC_OK && kept) st = ops_check_act(call, kept, ntok, dim);
    if (st == LC_OK && dx) st = ops_check_rows(call, "dx", dx, ntok, dim, true);
    if (st != LC_OK) return st;
    if ((x && x->dtype != dy->dtype) || (dx && dx->dtype != dy->dtype))
        return fail_status(LC_ERR_INVALID_ARG, "%s: x and dx have dy's type", call);
    if (!plain_params(weight, dim, w_dtype))
        return fail_status(LC_ERR_INVALID_ARG, "%s: weight is NULL, misaligned or of unknown dtype", call);
    if (ntok > 0 && (kind == LC_NORM_RMS) != (mean == nullptr))
        return fail_status(LC_ERR_INVALID_ARG, "%s: mean goes with LC_NORM_LAYER, and only with it", call);
    if (reinterpret_cast<uintptr_t>(mean) % 4 || reinterpret_cast<uintptr_t>(rstd) % 4)
        return fail_status(LC_ERR_INVALID_ARG, "%s: mean or rstd is not element-aligned", call);
    const int ge = elem_size(g_dtype);
    if (!ge || reinterpret_cast<uintptr_t>(dweight) % uintptr_t(ge) || reinterpret_cast<uintptr_t>(dbias) % uintptr_t(ge))
        return fail_status(LC_ERR_INVALID_ARG, "%s: dweight or dbias is misaligned or of unknown dtype", call);
    const bool want = dweight || dbias;
    const uint64_t need = want ? lc_norm_grad_workspace(ntok, dim) : 0;
    if (workspace_bytes < need)
        return fail_status(LC_ERR_CAPACITY, "%s: %llu bytes of workspace, %llu needed", call,
                           (unsigned long long)workspace_bytes, (unsigned long long)need);
    if (need && reinterpret_cast<uintptr_t>(workspace) % 256)
        return fail_status(LC_ERR_INVALID_ARG, "%s: the workspace is not 256-byte aligned", call);
    OnDevice cur(device);
    const int we = elem_size(w_dtype);
    const int64_t blocks = (dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    Span2 spans[10];
    int n = 0;
    spans[n++] = span_of("dy", dy, ntok, dim, false);
    if (x) spans[n++] = span_of("x", x, ntok, dim, false);
    if (kept) {
        spans[n++] = {"q", kept->q, ntok, blocks * LC_ACT_BLOCK, kept->q_stride, false};
        spans[n++] = {"e", kept->e, ntok, blocks, kept->e_stride, false};
    }
    spans[n++] = {"weight", weight, 1, dim * we, 0, false};
    if (mean) spans[n++] = {"mean", mean, 1, ntok * 4, 0, false};
    spans[n++] = {"rstd", rstd, 1, ntok * 4, 0, false};
    if (dx) spans[n++] = span_of("dx", dx, ntok, dim, true);
    if (dweight) spans[n++] = {"dweight", dweight, 1, dim * ge, 0, true};
    if (dbias) spans[n++] = {"dbias", dbias, 1, dim * ge, 0, true};
    if (need) spans[n++] = {"workspace", workspace, 1, int64_t(need), 0, true};
    st = ops_check(call, device, spans, n);
    if (st != LC_OK) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "%s: cannot make device %d current", call, device);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t err = cudaSuccess;
    if (ntok == 0) {
        if (accumulate) return LC_OK;
        if (dweight) err = cudaMemsetAsync(dweight, 0, size_t(dim * ge), s);
        if (err == cudaSuccess && dbias) err = cudaMemsetAsync(dbias, 0, size_t(dim * ge), s);
        return ops_launched(call, err);
    }
    NormGradParams p{};
    const int e = elem_size(dy->dtype);
    p.dy = static_cast<const uint8_t*>(dy->data);
    p.dy_pitch = dy->stride * e;
    if (x) {
        p.x = static_cast<const uint8_t*>(x->data);
        p.x_pitch = x->stride * e;
    } else {
        p.q = kept->q;
        p.e = kept->e;
        p.q_pitch = kept->q_stride;
        p.e_pitch = kept->e_stride;
    }
    p.w = static_cast<const uint8_t*>(weight);
    p.mean = mean;
    p.rstd = rstd;
    if (dx) {
        p.dx = static_cast<uint8_t*>(dx->data);
        p.dx_pitch = dx->stride * e;
    }
    p.part = static_cast<float*>(workspace);
    p.ntok = ntok;
    p.inv_dim = float(1.0 / double(dim));
    p.dim = int32_t(dim);
    p.w_bf16 = w_dtype == LC_BF16;
    p.rms = kind == LC_NORM_RMS;
    p.want_params = want;
    const bool vec = aligned16(p.dy) && aligned16(p.x) && aligned16(p.dx) && aligned16(p.w) && p.dy_pitch % 16 == 0 &&
                     p.x_pitch % 16 == 0 && p.dx_pitch % 16 == 0;
    const int sms = ops_sm_count(device);
    using B = __nv_bfloat16;
    int ctas = 0;
    if (dy->dtype == LC_BF16)
        err = x ? (vec ? dispatch_grad<B, true, false>(p, sms, s, &ctas) : dispatch_grad<B, false, false>(p, sms, s, &ctas))
                : (vec ? dispatch_grad<B, true, true>(p, sms, s, &ctas) : dispatch_grad<B, false, true>(p, sms, s, &ctas));
    else
        err = x ? (vec ? dispatch_grad<float, true, false>(p, sms, s, &ctas) : dispatch_grad<float, false, false>(p, sms, s, &ctas))
                : (vec ? dispatch_grad<float, true, true>(p, sms, s, &ctas) : dispatch_grad<float, false, true>(p, sms, s, &ctas));
    if (err == cudaSuccess && want) {
        FoldParams f{p.part, static_cast<uint8_t*>(dweight), static_cast<uint8_t*>(dbias), ctas, p.dim,
                     g_dtype == LC_BF16, accumulate != 0};
        cudaLaunchAttribute attr{};
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cudaLaunchConfig_t c{};
        c.gridDim = dim3(unsigned((dim + 31) / 32), dbias ? 2 : 1);
        c.blockDim = dim3(256);
        c.stream = s;
        c.attrs = &attr;
        c.numAttrs = 1;
        cudaGetLastError();
        err = cudaLaunchKernelEx(&c, norm_fold_kernel, f);
    }
    return ops_launched(call, err);
}
