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
//
// Rows whose addresses and length are multiples of 16 bytes (and not few and short)
// stream through shared memory: every group of threads has a ring of rows there, the
// next ones on their way by bulk copies while it works on one.  In registers as many
// bytes in flight would leave no room for the work: 16384 rows of 4096 bf16 through
// a root-mean-square norm 82 us that way, 48 so, their backward from the checkpoint 117 us
// and 67.
#include "lc_rows.cuh"

namespace lc {
namespace {

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
    int32_t stall;        // test switch: a ring's first copy announces 16 bytes that never come
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
    int32_t stall;        // as in NormParams
};

// The columns that a thread of a group of G holds: VPT vectors of V, 16 bytes each
// (VEC), or as many single elements G apart.
template <int V, int G, int VPT, bool VEC>
__device__ __forceinline__ int column(int t, int i, int j) {
    return VEC ? (i * G + t) * V + j : (i * V + j) * G + t;
}

// The thread's part of a row.  All vectors are asked for before the first is
// unpacked: in one loop each would be waited for in turn.
template <typename T, int G, int VPT, bool VEC>
__device__ __forceinline__ void load_row(const uint8_t* row, int t, int dim, float (&f)[VPT][kVec<T>]) {
    constexpr int V = kVec<T>;
    const T* r = reinterpret_cast<const T*>(row);
    uint4 raw[VPT];
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            if (column<V, G, VPT, VEC>(t, i, 0) + V <= dim) raw[i] = ld_stream(r + column<V, G, VPT, VEC>(t, i, 0));
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        if constexpr (VEC) unpack(raw[i], f[i]);
        if (!VEC || column<V, G, VPT, VEC>(t, i, 0) + V > dim) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int c = column<V, G, VPT, VEC>(t, i, j);
                f[i][j] = c < dim ? to_f32(r[c]) : 0.0f;
            }
        }
    }
}

// The i-th of the thread's vectors of a row.
template <typename T, int G, int VPT, bool VEC>
__device__ __forceinline__ void store_vec(uint8_t* row, int t, int i, int dim, const float (&f)[kVec<T>]) {
    constexpr int V = kVec<T>;
    T* r = reinterpret_cast<T*>(row);
    if (VEC && column<V, G, VPT, VEC>(t, i, 0) + V <= dim) {
        st_stream(r + column<V, G, VPT, VEC>(t, i, 0), pack(f));
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int c = column<V, G, VPT, VEC>(t, i, j);
            if (c < dim) r[c] = from_f32<T>(f[j]);
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

constexpr int cta_threads(int G) { return G < 128 ? 128 : G; }

template <typename T, int G, int VPT, bool VEC>
__global__ void __launch_bounds__(cta_threads(G)) norm_kernel(NormParams p) {
    constexpr int V = kVec<T>;
    constexpr int R = cta_threads(G) / G;   // rows of a CTA at a time
    __shared__ __align__(16) float shared[2][1][32];
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
            group_sum<G, cta_threads(G)>(s, shared, slot);
            mean = s[0] * p.inv_dim;
            s[0] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if (!VEC || column<V, G, VPT, VEC>(t, i, 0) + V > p.dim) {
                // what lies beyond the row is at the mean
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (column<V, G, VPT, VEC>(t, i, j) >= p.dim) f[i][j] = mean;
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                f[i][j] -= mean;
                s[0] = fmaf(f[i][j], f[i][j], s[0]);
            }
        }
        group_sum<G, cta_threads(G)>(s, shared, slot);
        const float rstd = rsqrtf(s[0] * p.inv_dim + p.eps);
        uint8_t* y = p.y + r * p.y_pitch;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if (VEC && column<V, G, VPT, VEC>(t, i, 0) >= p.dim) break;
            float w[V];
            load_param<V, G, VPT, VEC>(p.w, p.w_bf16, t, i, p.dim, w);
#pragma unroll
            for (int j = 0; j < V; ++j) f[i][j] *= rstd * w[j];
            if (p.b) {
                load_param<V, G, VPT, VEC>(p.b, p.w_bf16, t, i, p.dim, w);
#pragma unroll
                for (int j = 0; j < V; ++j) f[i][j] += w[j];
            }
            store_vec<T, G, VPT, VEC>(y, t, i, p.dim, f[i]);
        }
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
    dependents_may_start();
    __shared__ __align__(16) float shared[2][2][32];
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
            uint32_t w[VPT][V / 4];
            int code[VPT];
            if constexpr (VEC) {
                // V values of one block; a row ends with a whole block
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    const int c = column<V, G, VPT, VEC>(t, i, 0);
                    w[i][0] = code[i] = 0;
                    if (c >= p.dim) continue;
                    if constexpr (V == 8) {
                        const uint2 v = __ldcs(reinterpret_cast<const uint2*>(q + c));
                        w[i][0] = v.x;
                        w[i][1] = v.y;
                    } else {
                        w[i][0] = __ldcs(reinterpret_cast<const uint32_t*>(q + c));
                    }
                    code[i] = ex[c / LC_ACT_BLOCK];
                }
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if constexpr (VEC) {
                    const uint32_t s2 = act_scale2(code[i]);
#pragma unroll
                    for (int j = 0; j < V; j += 4) {
                        const uint2 v = act_values(w[i][j / 4], s2);
                        h[i][j] = __uint_as_float(v.x << 16);
                        h[i][j + 1] = __uint_as_float(v.x & 0xffff0000u);
                        h[i][j + 2] = __uint_as_float(v.y << 16);
                        h[i][j + 3] = __uint_as_float(v.y & 0xffff0000u);
                    }
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
        group_sum<G, cta_threads(G)>(s, shared, slot);
        if (p.dx) {
            const float m1 = p.rms ? 0.0f : s[0] * p.inv_dim, m2 = s[1] * p.inv_dim;
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) g[i][j] = rstd * (g[i][j] - m1 - h[i][j] * m2);
#pragma unroll
            for (int i = 0; i < VPT; ++i) store_vec<T, G, VPT, VEC>(p.dx + r * p.dx_pitch, t, i, p.dim, g[i]);
        }
    }
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

// --- rows through shared memory ---------------------------------------------------

constexpr int kFwdThreads = 1024;   // of a CTA, one a multiprocessor: 64 registers each (with 512: 55 us for 48)

template <typename T, int G, int VPT>
__global__ void __launch_bounds__(kFwdThreads, 1) norm_ring_kernel(NormParams p, int depth) {
    constexpr int V = kVec<T>, NT = kFwdThreads, R = NT / G;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float shared[2][1][32];
    __shared__ __align__(8) uint64_t bars[R * kRingMax];
    __shared__ uint32_t lost_by[NT / 32];
    volatile uint32_t& lost = lost_by[threadIdx.x >> 5];
    int slot = 0;
    const int t = threadIdx.x % G, group = threadIdx.x / G;
    float4* params = reinterpret_cast<float4*>(smem);
    constexpr int kParam = VPT * V / 4 * G;
    RowRing ring;
    ring.bytes = uint32_t(p.dim) * uint32_t(sizeof(T));
    ring.depth = depth;
    ring.data = smem_addr(smem) + kParam * 16 * (p.b ? 2 : 1) + group * depth * ring.bytes;
    ring.bar = smem_addr(bars) + group * kRingMax * 8;
    if (threadIdx.x < R * kRingMax) {
        mbar_init(smem_addr(bars) + 8 * threadIdx.x, 1);
        mbar_init_fence();
    }
    lost = 0;
    __syncthreads();
    // rows of the group: consecutive ones go to different CTAs
    const int64_t step = int64_t(gridDim.x) * R;
    int64_t r = int64_t(group) * gridDim.x + blockIdx.x;
    int64_t ahead = r;           // first row not asked for
    if (t == 0)
        for (int i = 0; i < depth && ahead < p.ntok; ++i, ahead += step) {
            mbar_expect_tx(ring.bar + 8 * i, ring.bytes + (i == 0 && p.stall ? 16 : 0));
            bulk_g2s(ring.data + i * ring.bytes, p.x + ahead * p.x_pitch, ring.bytes, ring.bar + 8 * i);
        }
    stage_param<V, G, VPT>(params, p.w, p.w_bf16, p.dim, NT);
    if (p.b) stage_param<V, G, VPT>(params + kParam, p.b, p.w_bf16, p.dim, NT);
    __syncthreads();
    for (; r < p.ntok; r += step) {
        const bool ok = ring_wait(ring, lost);
        float f[VPT][V];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (i * G + t) * V;
            if (c < p.dim) {
                unpack(lds128(ring.row() + c * int(sizeof(T))), f[i]);
                if (!ok) f[i][0] = __uint_as_float(0x7fffffffu);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) f[i][j] = 0.0f;
            }
        }
        // the row has been read by all once they met in a sum
        auto refill = [&]() {
            if (t == 0 && ahead < p.ntok && !lost) {
                mbar_expect_tx(ring.full(), ring.bytes);
                bulk_g2s(ring.row(), p.x + ahead * p.x_pitch, ring.bytes, ring.full());
            }
            ahead += step;
            ring.next();
        };
        if (p.q) {
            constexpr int L = LC_ACT_BLOCK / V;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                float amax = 0.0f;
#pragma unroll
                for (int j = 0; j < V; ++j) amax = max_nan(amax, f[i][j]);
                const int code = act_code(block_amax<L>(amax));
                const int c = (i * G + t) * V;
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
        float s[1] = {0.0f};
        float mean = 0.0f;
        float part[4] = {};          // short chains
        if (!p.rms) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int j = 0; j < V; ++j) part[j & 3] += f[i][j];
            s[0] = (part[0] + part[1]) + (part[2] + part[3]);
            group_sum<G, NT>(s, shared, slot);
            refill();
            mean = s[0] * p.inv_dim;
            part[0] = part[1] = part[2] = part[3] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if ((i * G + t) * V >= p.dim) break;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                f[i][j] -= mean;
                part[j & 3] = fmaf(f[i][j], f[i][j], part[j & 3]);
            }
        }
        s[0] = (part[0] + part[1]) + (part[2] + part[3]);
        group_sum<G, NT>(s, shared, slot);
        if (p.rms) refill();
        const float rstd = rsqrtf(s[0] * p.inv_dim + p.eps);
        T* y = reinterpret_cast<T*>(p.y + r * p.y_pitch);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (i * G + t) * V;
            if (c >= p.dim) break;
#pragma unroll
            for (int j = 0; j < V; j += 4) {
                const float4 w = params[(i * (V / 4) + j / 4) * G + t];
                float4 b = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (p.b) b = params[kParam + (i * (V / 4) + j / 4) * G + t];
                f[i][j] = fmaf(f[i][j], rstd * w.x, b.x);
                f[i][j + 1] = fmaf(f[i][j + 1], rstd * w.y, b.y);
                f[i][j + 2] = fmaf(f[i][j + 2], rstd * w.z, b.z);
                f[i][j + 3] = fmaf(f[i][j + 3], rstd * w.w, b.w);
            }
            st_stream(y + c, pack(f[i]));
        }
        if (t == 0) {
            if (!p.rms) p.mean[r] = mean;
            p.rstd[r] = rstd;
        }
    }
    ring_drain(ring, lost, t);
}

constexpr int kBwdThreads = 512;    // 128 registers each: sums for weight and bias besides the row (before the
                                    // arithmetic in pairs 77 us; 8 values a thread and 1024 threads 104, 32 values and 384 threads 75)

// The backward.  A slot holds the rows of dy and of x (or its 8-bit values; their
// exponents are asked for a row ahead into registers).
// LEAN: no means (root-mean-square norm) and no gradient of a bias.
template <typename T, int G, int VPT, bool KEPT, bool LEAN>
__global__ void __launch_bounds__(kBwdThreads, 1) norm_grad_ring_kernel(NormGradParams p, int depth) {
    constexpr int V = kVec<T>, NT = kBwdThreads, R = NT / G;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(16) float shared[2][2][32];
    float(*shared1)[1][32] = reinterpret_cast<float(*)[1][32]>(shared);
    __shared__ __align__(8) uint64_t bars[R * kRingMax];
    __shared__ uint32_t lost_by[NT / 32];
    volatile uint32_t& lost = lost_by[threadIdx.x >> 5];
    dependents_may_start();
    int slot = 0;
    const int t = threadIdx.x % G, group = threadIdx.x / G;
    float4* params = reinterpret_cast<float4*>(smem);
    constexpr int kParam = VPT * V / 4 * G;
    const uint32_t dy_bytes = uint32_t(p.dim) * uint32_t(sizeof(T));
    const uint32_t x_bytes = KEPT ? uint32_t(p.dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK * LC_ACT_BLOCK : dy_bytes;
    RowRing ring;
    ring.bytes = dy_bytes + x_bytes;
    ring.depth = depth;
    ring.data = smem_addr(smem) + kParam * 16 + group * depth * ring.bytes;
    ring.bar = smem_addr(bars) + group * kRingMax * 8;
    if (threadIdx.x < R * kRingMax) {
        mbar_init(smem_addr(bars) + 8 * threadIdx.x, 1);
        mbar_init_fence();
    }
    lost = 0;
    __syncthreads();
    const int64_t step = int64_t(gridDim.x) * R;
    int64_t r = int64_t(group) * gridDim.x + blockIdx.x;
    int64_t ahead = r;
    auto fetch = [&](int at, uint32_t more) {
        const uint32_t to = ring.data + at * ring.bytes, bar = ring.bar + 8 * at;
        mbar_expect_tx(bar, ring.bytes + more);
        bulk_g2s(to, p.dy + ahead * p.dy_pitch, dy_bytes, bar);
        bulk_g2s(to + dy_bytes, KEPT ? reinterpret_cast<const uint8_t*>(p.q) + ahead * p.q_pitch : p.x + ahead * p.x_pitch, x_bytes, bar);
    };
    if (t == 0)
        for (int i = 0; i < depth && ahead < p.ntok; ++i, ahead += step) fetch(i, i == 0 && p.stall ? 16 : 0);
    stage_param<V, G, VPT>(params, p.w, p.w_bf16, p.dim, NT);
    __syncthreads();
    float2 dw[VPT][V / 2], db[LEAN ? 1 : VPT][V / 2];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V / 2; ++j) dw[i][j] = db[LEAN ? 0 : i][j] = both(0.0f);
    int code[VPT];
    float mean = 0.0f, rstd = 0.0f;
    auto row_values = [&](int64_t at) {   // what a row has beside its vectors
        if (at >= p.ntok) return;
        if (!LEAN && !p.rms) mean = __ldg(p.mean + at);
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
    for (; r < p.ntok; r += step) {
        const bool ok = ring_wait(ring, lost);
        float2 a[VPT][V / 2], h[VPT][V / 2];   // dy, then dy w; x, then its normalised value
        const float mu = mean, rs = ok ? rstd : __uint_as_float(0x7fffffffu);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (i * G + t) * V;
            if (c >= p.dim) break;
            unpack(lds128(ring.row() + c * int(sizeof(T))), a[i]);
            if constexpr (KEPT) {
                const uint32_t at = ring.row() + dy_bytes + c;
                uint32_t q[V / 4];
                if constexpr (V == 8) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(q[0]), "=r"(q[1]) : "r"(at) : "memory");
                else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(q[0]) : "r"(at) : "memory");
                // a byte + 128 in the fraction of 2^23 gives its value; the product with the scale is exact
                const float sc = act_scale(code[i]);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    const uint32_t w = q[j / 2] ^ 0x80808080u;
                    const int b = j & 1 ? 2 : 0;
                    const float2 u = make_float2(__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7650 | b)),
                                                 __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7651 | b)));
                    const float2 v = add2(u, both(-8388736.0f));
                    if constexpr (LEAN) h[i][j] = mul2(v, both(sc * rs));
                    else h[i][j] = mul2(fma2(v, both(sc), both(-mu)), both(rs));
                }
            } else {
                unpack(lds128(ring.row() + dy_bytes + c * int(sizeof(T))), h[i]);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    if constexpr (!LEAN) h[i][j] = add2(h[i][j], both(-mu));
                    h[i][j] = mul2(h[i][j], both(rs));
                }
            }
        }
        row_values(r + step);
        float s[2] = {0.0f, 0.0f};
        float2 s0[2] = {both(0.0f), both(0.0f)}, s1[2] = {both(0.0f), both(0.0f)};   // short chains
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
                    if constexpr (!LEAN) db[i][j + m] = add2(db[i][j + m], a[i][j + m]);
                    a[i][j + m] = mul2(a[i][j + m], w[m]);
                    if constexpr (!LEAN) s0[m] = add2(s0[m], a[i][j + m]);
                    s1[m] = fma2(a[i][j + m], h[i][j + m], s1[m]);
                }
            }
        }
        s0[0] = add2(s0[0], s0[1]);
        s1[0] = add2(s1[0], s1[1]);
        s[0] = s0[0].x + s0[0].y;
        s[1] = s1[0].x + s1[0].y;
        if constexpr (LEAN) {
            float one[1] = {s[1]};
            group_sum<G, NT>(one, shared1, slot);
            s[1] = one[0];
        } else {
            group_sum<G, NT>(s, shared, slot);
        }
        if constexpr (G == 32) __syncwarp();
        if (t == 0 && ahead < p.ntok && !lost) fetch(ring.at, 0);
        ahead += step;
        ring.next();
        if (p.dx) {
            const float m1 = LEAN || p.rms ? 0.0f : s[0] * p.inv_dim * rs, m2 = s[1] * p.inv_dim * rs;
            T* dx = reinterpret_cast<T*>(p.dx + r * p.dx_pitch);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int c = (i * G + t) * V;
                if (c >= p.dim) break;
#pragma unroll
                for (int j = 0; j < V / 2; ++j) {
                    const float2 v = LEAN ? mul2(a[i][j], both(rs)) : fma2(a[i][j], both(rs), both(-m1));
                    a[i][j] = fma2(h[i][j], both(-m2), v);
                }
                st_stream(dx + c, pack(a[i]));
            }
        }
    }
    ring_drain(ring, lost, t);
    if (!p.want_params) return;
    if (lost) {
        // NaN came into dw with h; db has added up whatever was in the row's place
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < V / 2; ++j) dw[i][j] = db[LEAN ? 0 : i][j] = both(__uint_as_float(0x7fffffffu));
    }
    // one row of sums for the CTA: every group leaves its own in the rings' memory (all rows were read), and each
    // column is added over the groups in order
    float* out = p.part + int64_t(blockIdx.x) * 2 * p.dim;
    auto quad = [](const float2& x, const float2& y) { return make_float4(x.x, x.y, y.x, y.y); };
    if constexpr (R == 1) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int c = (i * G + t) * V;
            if (c >= p.dim) break;
#pragma unroll
            for (int j = 0; j < V / 2; j += 2) {
                *reinterpret_cast<float4*>(out + c + 2 * j) = quad(dw[i][j], dw[i][j + 1]);
                if constexpr (!LEAN) *reinterpret_cast<float4*>(out + p.dim + c + 2 * j) = quad(db[i][j], db[i][j + 1]);
            }
        }
    } else {
        __syncthreads();
        constexpr int kCols = VPT * V * G;
        float4* sums = reinterpret_cast<float4*>(smem);   // [groups][dw, db][VPT * V / 4][G]
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < V / 2; j += 2) {
                float4* at = sums + group * (kCols / 2) + (i * (V / 4) + j / 2) * G + t;
                at[0] = quad(dw[i][j], dw[i][j + 1]);
                if constexpr (!LEAN) at[kCols / 4] = quad(db[i][j], db[i][j + 1]);
            }
        __syncthreads();
        for (int k = threadIdx.x; k < kCols / (LEAN ? 4 : 2); k += NT) {
            const int q = k % (kCols / 4);
            const int c = (q / G / (V / 4) * G + q % G) * V + q / G % (V / 4) * 4;
            if (c >= p.dim) continue;
            float4 v = sums[k];
#pragma unroll 4
            for (int g = 1; g < R; ++g) {
                const float4 x = sums[g * (kCols / 2) + k];
                v.x += x.x;
                v.y += x.y;
                v.z += x.z;
                v.w += x.w;
            }
            *reinterpret_cast<float4*>(out + (k < kCols / 4 ? 0 : p.dim) + c) = v;
        }
    }
}

struct FoldParams {
    const float* part;
    uint8_t* dw;
    uint8_t* db;
    int32_t rows, dim, g_bf16, accumulate;
};

// Adds the CTAs' rows of sums: 32 columns a CTA, a warp every 32nd row, the warps'
// sums added in order.
__global__ void __launch_bounds__(1024) norm_fold_kernel(FoldParams p) {
    __shared__ float sums[32][33];
    dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    uint8_t* out = blockIdx.y ? p.db : p.dw;
    if (!out) return;
    const float* part = p.part + (blockIdx.y ? p.dim : 0);
    float s = 0.0f;
    if (c < p.dim) {
#pragma unroll 4
        for (int r = warp; r < p.rows; r += 32) s += part[int64_t(r) * 2 * p.dim + c];
    }
    sums[warp][lane] = s;
    __syncthreads();
    if (warp || c >= p.dim) return;
#pragma unroll
    for (int i = 1; i < 32; ++i) s += sums[i][lane];
    if (p.g_bf16) {
        __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(out) + c;
        *o = __float2bfloat16_rn(p.accumulate ? __bfloat162float(*o) + s : s);
    } else {
        float* o = reinterpret_cast<float*>(out) + c;
        *o = p.accumulate ? *o + s : s;
    }
}

template <typename T, int G, int VPT>
cudaError_t launch_norm_ring(const NormParams& p, int sms, cudaStream_t s, bool* done) {
    constexpr int V = kVec<T>, NT = kFwdThreads, R = NT / G;
    if (p.dim > G * VPT * V) return cudaErrorInvalidValue;   // every column has a thread
    static bool ready[kOpsMaxDevices];
    const size_t params = size_t(VPT) * V * G * 4 * (p.b ? 2 : 1), row = size_t(p.dim) * sizeof(T);
    const int depth = ring_depth(params, R, row);
    *done = depth > 0;
    if (!depth) return cudaSuccess;
    const cudaError_t e = allow_smem(norm_ring_kernel<T, G, VPT>, ready);
    if (e != cudaSuccess) return e;
    const int64_t grid = p.ntok < sms ? p.ntok : sms;
    cudaGetLastError();
    norm_ring_kernel<T, G, VPT><<<unsigned(grid), NT, params + R * depth * row, s>>>(p, depth);
    return cudaGetLastError();
}

template <typename T>
cudaError_t dispatch_norm_ring(const NormParams& p, int sms, cudaStream_t s, bool* done) {
    constexpr int M = 8 / kVec<T>;          // 16 values a thread, from a warp a row on
    const int nv = (p.dim / kVec<T> + M - 1) / M;   // an fp32 row may end half way through its last 8 values
    if (nv <= 32) return launch_norm_ring<T, 32, M>(p, sms, s, done);
    if (nv <= 64) return launch_norm_ring<T, 32, 2 * M>(p, sms, s, done);
    if (nv <= 96) return launch_norm_ring<T, 32, 3 * M>(p, sms, s, done);
    if (nv <= 128) return launch_norm_ring<T, 64, 2 * M>(p, sms, s, done);
    if (nv <= 256) return launch_norm_ring<T, 128, 2 * M>(p, sms, s, done);
    if (nv <= 512) return launch_norm_ring<T, 256, 2 * M>(p, sms, s, done);
    if (nv <= 1024) return launch_norm_ring<T, 512, 2 * M>(p, sms, s, done);
    return launch_norm_ring<T, 1024, 2 * M>(p, sms, s, done);
}

template <typename T, int G, int VPT, bool KEPT, bool LEAN>
cudaError_t launch_grad_ring(const NormGradParams& p, int sms, cudaStream_t s, int* ctas) {
    constexpr int V = kVec<T>, NT = kBwdThreads, R = NT / G;
    if (p.dim > G * VPT * V) return cudaErrorInvalidValue;   // every column has a thread
    static bool ready[kOpsMaxDevices];
    const size_t params = size_t(VPT) * V * G * 4;
    const size_t row = size_t(p.dim) * sizeof(T) + (KEPT ? (size_t(p.dim) + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK * LC_ACT_BLOCK
                                                         : size_t(p.dim) * sizeof(T));
    const int depth = ring_depth(params, R, row);
    *ctas = 0;
    if (!depth) return cudaSuccess;
    const cudaError_t e = allow_smem(norm_grad_ring_kernel<T, G, VPT, KEPT, LEAN>, ready);
    if (e != cudaSuccess) return e;
    int64_t grid = p.ntok < sms ? p.ntok : sms;
    grid = grid < kGradCtas ? grid : kGradCtas;
    *ctas = int(grid);
    size_t smem = params + R * depth * row;
    if (R > 1 && smem < 2 * R * params) smem = 2 * R * params;   // the groups' sums
    cudaGetLastError();
    norm_grad_ring_kernel<T, G, VPT, KEPT, LEAN><<<unsigned(grid), NT, smem, s>>>(p, depth);
    return cudaGetLastError();
}

template <typename T, bool KEPT, bool LEAN>
cudaError_t dispatch_grad_ring(const NormGradParams& p, int sms, cudaStream_t s, int* ctas) {
    constexpr int M = 8 / kVec<T>;
    const int nv = (p.dim / kVec<T> + M - 1) / M;   // an fp32 row may end half way through its last 8 values
    if (nv <= 32) return launch_grad_ring<T, 32, M, KEPT, LEAN>(p, sms, s, ctas);
    if (nv <= 64) return launch_grad_ring<T, 32, 2 * M, KEPT, LEAN>(p, sms, s, ctas);
    if (nv <= 96) return launch_grad_ring<T, 32, 3 * M, KEPT, LEAN>(p, sms, s, ctas);
    if (nv <= 128) return launch_grad_ring<T, 64, 2 * M, KEPT, LEAN>(p, sms, s, ctas);
    if (nv <= 256) return launch_grad_ring<T, 128, 2 * M, KEPT, LEAN>(p, sms, s, ctas);
    if (nv <= 512) return launch_grad_ring<T, 256, 2 * M, KEPT, LEAN>(p, sms, s, ctas);
    if (nv <= 1024) return launch_grad_ring<T, 512, 2 * M, KEPT, LEAN>(p, sms, s, ctas);
    return launch_grad_ring<T, 512, 4 * M, KEPT, LEAN>(p, sms, s, ctas);
}

template <typename T, int G, int VPT, bool VEC>
cudaError_t launch_norm(const NormParams& p, int sms, cudaStream_t s) {
    constexpr int R = cta_threads(G) / G;
    const int64_t want = (p.ntok + R - 1) / R;
    const int64_t most = int64_t(sms) * 1024;
    cudaGetLastError();
    norm_kernel<T, G, VPT, VEC><<<unsigned(want < most ? want : most), cta_threads(G), 0, s>>>(p);
    return cudaGetLastError();
}

// Threads of a row and vectors of a thread: a warp up to 4 vectors a lane, then
// groups of warps.
template <typename T, bool VEC>
cudaError_t dispatch_norm(const NormParams& p, int sms, cudaStream_t s) {
    const int nv = (p.dim + kVec<T> - 1) / kVec<T>;
    if (nv <= 32) return launch_norm<T, 32, 1, VEC>(p, sms, s);
    if (nv <= 64) return launch_norm<T, 32, 2, VEC>(p, sms, s);
    if (nv <= 128) return launch_norm<T, 32, 4, VEC>(p, sms, s);
    if (nv <= 256) return launch_norm<T, 128, 2, VEC>(p, sms, s);
    if (nv <= 512) return launch_norm<T, 128, 4, VEC>(p, sms, s);
    if (nv <= 1024) return launch_norm<T, 256, 4, VEC>(p, sms, s);
    if constexpr (kVec<T> == 4)
        if (nv > 2048) return launch_norm<T, 1024, 4, VEC>(p, sms, s);
    return launch_norm<T, 512, 4, VEC>(p, sms, s);
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

// Whether the rings pay (microseconds through them and directly; bf16 but for the last):
//   forward    64 rows of 768: 3.1, 3.7; 2432 of 4096: 9.8, 14.3; 2432 of 256: 3.1, 2.7
//   backward   64 of 4096: 6.4, 8.9; 152 of 768: 6.0, 5.2; 304 of 768: 6.2, 7.1; 608 of 256: 5.2, 4.5; 1216 of 256:
//              5.2, 5.6; fp32 152 of 1024: 5.8, 4.7; 304 of 1024: 5.8, 6.2
bool forward_ring(int64_t ntok, int64_t row_bytes) { return row_bytes >= 1024 || ntok >= 4096; }
bool backward_ring(int64_t ntok, int64_t row_bytes, int sms) {
    return row_bytes >= 8192 || ntok >= (row_bytes >= 1024 ? 2 * sms : 1024);
}
constexpr int64_t kMaxRows = int64_t(1) << 40;

bool plain_params(const void* w, int64_t dim, int32_t dtype) {
    return w && elem_size(dtype) && reinterpret_cast<uintptr_t>(w) % uintptr_t(elem_size(dtype)) == 0 && dim > 0;
}

}  // namespace

cudaError_t norm_fold(const float* part, int rows, int dim, void* dw, void* db, bool bf16, bool accumulate, cudaStream_t s) {
    const FoldParams f{part, static_cast<uint8_t*>(dw), static_cast<uint8_t*>(db), rows, dim, bf16, accumulate};
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(unsigned((dim + 31) / 32), db ? 2 : 1);
    c.blockDim = dim3(1024);
    c.stream = s;
    c.attrs = &attr;
    c.numAttrs = 1;
    cudaGetLastError();
    return cudaLaunchKernelEx(&c, norm_fold_kernel, f);
}

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
    p.stall = ops_stall();
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
    cudaError_t err = cudaSuccess;
    bool done = false;
    if (vec && dim * e % 16 == 0 && forward_ring(ntok, dim * e))
        err = x->dtype == LC_BF16 ? dispatch_norm_ring<__nv_bfloat16>(p, sms, s, &done) : dispatch_norm_ring<float>(p, sms, s, &done);
    if (done || err != cudaSuccess) return ops_launched(call, err);
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
    p.stall = ops_stall();
    const bool vec = aligned16(p.dy) && aligned16(p.x) && aligned16(p.dx) && aligned16(p.w) && p.dy_pitch % 16 == 0 &&
                     p.x_pitch % 16 == 0 && p.dx_pitch % 16 == 0;
    const int sms = ops_sm_count(device);
    using B = __nv_bfloat16;
    int ctas = 0;
    if (vec && dim * e % 16 == 0 && backward_ring(ntok, dim * e, sms)) {
        const bool lean = kind == LC_NORM_RMS && !dbias, bf = dy->dtype == LC_BF16;
        auto go = [&](auto f) { err = f(p, sms, s, &ctas); };
        if (bf && x) go(lean ? dispatch_grad_ring<B, false, true> : dispatch_grad_ring<B, false, false>);
        else if (bf) go(lean ? dispatch_grad_ring<B, true, true> : dispatch_grad_ring<B, true, false>);
        else if (x) go(lean ? dispatch_grad_ring<float, false, true> : dispatch_grad_ring<float, false, false>);
        else go(lean ? dispatch_grad_ring<float, true, true> : dispatch_grad_ring<float, true, false>);
    }
    if (ctas || err != cudaSuccess) {
        // through the rings
    } else if (dy->dtype == LC_BF16)
        err = x ? (vec ? dispatch_grad<B, true, false>(p, sms, s, &ctas) : dispatch_grad<B, false, false>(p, sms, s, &ctas))
                : (vec ? dispatch_grad<B, true, true>(p, sms, s, &ctas) : dispatch_grad<B, false, true>(p, sms, s, &ctas));
    else
        err = x ? (vec ? dispatch_grad<float, true, false>(p, sms, s, &ctas) : dispatch_grad<float, false, false>(p, sms, s, &ctas))
                : (vec ? dispatch_grad<float, true, true>(p, sms, s, &ctas) : dispatch_grad<float, false, true>(p, sms, s, &ctas));
    if (err == cudaSuccess && want) {
        err = norm_fold(p.part, ctas, p.dim, dweight, dbias, g_dtype == LC_BF16, accumulate != 0, s);
    }
    return ops_launched(call, err);
}
