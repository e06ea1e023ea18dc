// lc_act.cu -- activations in 8 bits: whole numbers of [-127, 127] with one power
// of two for a block of 128 values of a token.
//
// A power of two and not amax / 127: the value q * 2^e then is exactly a bf16
// number (seven bits of significand and a sign), so the products of the backward
// pass can take it as a tensor core operand without a rounding of their own, and
// the scale itself is one byte.  The price is at most one bit of the eight.
//
// Bound by memory: save reads 2 or 4 bytes a value and writes 1 + 1/128, load the
// other way round.
#include "lc_ops.cuh"

namespace lc {
namespace {

constexpr int kActThreads = 256;

struct ActParams {
    const uint8_t* x;     // save: rows in; load: rows out
    int8_t* q;
    int8_t* e;
    int64_t ntok, dim, blocks, x_pitch, q_pitch, e_pitch;
    int64_t items, segs;  // items = ntok * segs (segments of a row)
};

constexpr int kUnroll = 4;   // vectors that a lane has in flight

// A warp keeps a segment of a row.  VEC: kUnroll vectors of 16 bytes a lane, a
// block in 128 / V neighbouring lanes; otherwise kUnroll blocks, a lane every 32nd
// value of each.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kActThreads, 6) act_save_kernel(ActParams p) {
    constexpr int V = VEC ? kVec<T> : 4, L = VEC ? LC_ACT_BLOCK / V : 32;
    const int lane = threadIdx.x & 31;
    const int64_t item = int64_t(blockIdx.x) * (kActThreads / 32) + (threadIdx.x >> 5);
    if (item >= p.items) return;
    int64_t t, seg;
    split_item(item, p.segs, t, seg);
    const T* x = reinterpret_cast<const T*>(p.x + t * p.x_pitch);
    int8_t* q = p.q + t * p.q_pitch;
    const int64_t c0 = seg * (32 * V * kUnroll), padded = p.blocks * LC_ACT_BLOCK;
    float f[kUnroll][V];
    if constexpr (VEC) {
        uint4 v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t c = c0 + (u * 32 + lane) * V;
            if (c + V <= p.dim) v[u] = ld_stream(x + c);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t c = c0 + (u * 32 + lane) * V;
            unpack(v[u], f[u]);
            if (c + V > p.dim) {
#pragma unroll
                for (int i = 0; i < V; ++i) f[u][i] = c + i < p.dim ? to_f32(x[c + i]) : 0.0f;
            }
        }
    } else {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int64_t c = c0 + u * LC_ACT_BLOCK + i * 32 + lane;
                f[u][i] = c < p.dim ? to_f32(x[c]) : 0.0f;
            }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) amax = max_nan(amax, f[u][i]);
        const int code = act_code(block_amax<L>(amax));
        uint32_t w[V / 4];
        act_bytes<V>(f[u], code, w);
        const int64_t c = c0 + (VEC ? (u * 32 + lane) * V : u * LC_ACT_BLOCK);
        if (c >= padded) break;
        if constexpr (!VEC) {
#pragma unroll
            for (int i = 0; i < 4; ++i) q[c + i * 32 + lane] = int8_t(w[0] >> (8 * i));
        } else if constexpr (V == 8) {
            *reinterpret_cast<uint2*>(q + c) = make_uint2(w[0], w[1]);
        } else {
            *reinterpret_cast<uint32_t*>(q + c) = w[0];
        }
        if (lane % L == 0) p.e[t * p.e_pitch + c / LC_ACT_BLOCK] = int8_t(code);
    }
}

// A warp gives a segment of a row: kUnroll times 8 values a lane (VEC), or
// kUnroll blocks, every 32nd value.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kActThreads) act_load_kernel(ActParams p) {
    constexpr int V = VEC ? 8 : 4;
    const int lane = threadIdx.x & 31;
    const int64_t item = int64_t(blockIdx.x) * (kActThreads / 32) + (threadIdx.x >> 5);
    if (item >= p.items) return;
    int64_t t, seg;
    split_item(item, p.segs, t, seg);
    T* x = reinterpret_cast<T*>(const_cast<uint8_t*>(p.x) + t * p.x_pitch);
    const int8_t* q = p.q + t * p.q_pitch;
    const int8_t* e = p.e + t * p.e_pitch;
    const int64_t c0 = seg * (32 * V * kUnroll);
    if constexpr (VEC) {
        uint2 w[kUnroll];
        int code[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t c = c0 + (u * 32 + lane) * V;
            if (c >= p.dim) break;
            w[u] = __ldcs(reinterpret_cast<const uint2*>(q + c));   // a row ends with a whole block
            code[u] = e[c / LC_ACT_BLOCK];
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t c = c0 + (u * 32 + lane) * V;
            if (c >= p.dim) break;
            const uint32_t s = act_scale2(code[u]);
            const uint2 a = act_values(w[u].x, s), b = act_values(w[u].y, s);
            const uint4 v = make_uint4(a.x, a.y, b.x, b.y);
            if (c + V <= p.dim) {
                if constexpr (sizeof(T) == 2) {
                    st_stream(x + c, v);
                } else {
                    float f[8];
                    unpack(v, f);
                    st_stream(x + c, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
                    st_stream(x + c + 4, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
                }
            } else {
                float f[8];
                unpack(v, f);
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (c + i < p.dim) x[c + i] = from_f32<T>(f[i]);
            }
        }
    } else {
        int v[kUnroll][V], code[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t c = c0 + u * LC_ACT_BLOCK;
            if (c >= p.dim) break;
            code[u] = e[c / LC_ACT_BLOCK];
#pragma unroll
            for (int i = 0; i < V; ++i) v[u][i] = q[c + i * 32 + lane];
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t c = c0 + u * LC_ACT_BLOCK + lane;
            const float s = act_scale(code[u]);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (c + i * 32 < p.dim) x[c + i * 32] = from_f32<T>(float(v[u][i]) * s);
        }
    }
}

// `per`: values of a segment.
template <typename K>
cudaError_t launch_act(K kernel, ActParams p, int64_t per, cudaStream_t s) {
    p.segs = (p.dim + per - 1) / per;
    p.items = p.ntok * p.segs;
    const int64_t grid = (p.items + kActThreads / 32 - 1) / (kActThreads / 32);
    if (grid > 0x7fffffff) return cudaErrorInvalidValue;
    cudaGetLastError();
    kernel<<<unsigned(grid), kActThreads, 0, s>>>(p);
    return cudaGetLastError();
}

ActParams act_params(const lc_rows* x, const lc_act* a, int64_t ntok, int64_t dim) {
    ActParams p{};
    p.x = static_cast<const uint8_t*>(x->data);
    p.q = a->q;
    p.e = a->e;
    p.ntok = ntok;
    p.dim = dim;
    p.blocks = (dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    p.x_pitch = x->stride * elem_size(x->dtype);
    p.q_pitch = a->q_stride;
    p.e_pitch = a->e_stride;
    return p;
}

lc_status check(const char* call, int device, const lc_rows* x, const char* name, const lc_act* a, int64_t ntok,
                int64_t dim, bool save) {
    if (ntok < 0 || dim <= 0 || ntok > (int64_t(1) << 40) || dim > (int64_t(1) << 40))
        return fail_status(LC_ERR_INVALID_ARG, "%s: %lld rows of %lld", call, (long long)ntok, (long long)dim);
    lc_status st = ops_check_rows(call, name, x, ntok, dim, !save);
    if (st == LC_OK) st = ops_check_act(call, a, ntok, dim);
    if (st != LC_OK) return st;
    const int64_t blocks = (dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    const Span2 spans[] = {span_of(name, x, ntok, dim, !save),
                           {"q", a->q, ntok, blocks * LC_ACT_BLOCK, a->q_stride, save},
                           {"e", a->e, ntok, blocks, a->e_stride, save}};
    return ops_check(call, device, spans, 3);
}

}  // namespace

cudaError_t act_save_rows(const lc_rows* x, const lc_act* a, int64_t ntok, int64_t dim, cudaStream_t s) {
    const ActParams p = act_params(x, a, ntok, dim);
    const bool vec = aligned16(x->data) && p.x_pitch % 16 == 0;
    using B = __nv_bfloat16;
    if (x->dtype == LC_BF16)
        return vec ? launch_act(act_save_kernel<B, true>, p, 32 * 8 * kUnroll, s)
                   : launch_act(act_save_kernel<B, false>, p, 32 * 4 * kUnroll, s);
    return vec ? launch_act(act_save_kernel<float, true>, p, 32 * 4 * kUnroll, s)
               : launch_act(act_save_kernel<float, false>, p, 32 * 4 * kUnroll, s);
}

}  // namespace lc

using namespace lc;

extern "C" lc_status lc_act_save(int device, void* cuda_stream, const lc_rows* x, int64_t ntok, int64_t dim,
                                 const lc_act* act) {
    set_last_error("");
    OnDevice cur(device);
    const lc_status st = check("lc_act_save", device, x, "x", act, ntok, dim, true);
    if (st != LC_OK || ntok == 0) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "lc_act_save: cannot make device %d current", device);
    return ops_launched("lc_act_save", act_save_rows(x, act, ntok, dim, static_cast<cudaStream_t>(cuda_stream)));
}

extern "C" lc_status lc_act_load(int device, void* cuda_stream, const lc_act* act, int64_t ntok, int64_t dim,
                                 const lc_rows* y) {
    set_last_error("");
    OnDevice cur(device);
    const lc_status st = check("lc_act_load", device, y, "y", act, ntok, dim, false);
    if (st != LC_OK || ntok == 0) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "lc_act_load: cannot make device %d current", device);
    const ActParams p = act_params(y, act, ntok, dim);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool vec = aligned16(y->data) && p.x_pitch % 16 == 0;
    using B = __nv_bfloat16;
    cudaError_t e;
    if (y->dtype == LC_BF16)
        e = vec ? launch_act(act_load_kernel<B, true>, p, 32 * 8 * kUnroll, s)
                : launch_act(act_load_kernel<B, false>, p, 32 * 4 * kUnroll, s);
    else
        e = vec ? launch_act(act_load_kernel<float, true>, p, 32 * 8 * kUnroll, s)
                : launch_act(act_load_kernel<float, false>, p, 32 * 4 * kUnroll, s);
    return ops_launched("lc_act_load", e);
}
