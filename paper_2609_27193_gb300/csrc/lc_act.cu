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
    int64_t items, segs;  // items = ntok * segs
};

// A warp keeps one block, four values a lane.  VEC: 4 consecutive values (8- or
// 16-byte loads); otherwise every 32nd, element by element.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kActThreads) act_save_kernel(ActParams p) {
    const int lane = threadIdx.x & 31;
    const int64_t step = int64_t(gridDim.x) * (kActThreads / 32);
    for (int64_t item = int64_t(blockIdx.x) * (kActThreads / 32) + (threadIdx.x >> 5); item < p.items; item += step) {
        const int64_t t = item / p.blocks, b = item - t * p.blocks;
        const T* x = reinterpret_cast<const T*>(p.x + t * p.x_pitch);
        const int64_t c0 = b * LC_ACT_BLOCK;
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t c = c0 + (VEC ? lane * 4 + i : i * 32 + lane);
            f[i] = c < p.dim ? to_f32(x[c]) : 0.0f;
        }
        float amax = 0.0f;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            amax = fmaxf(amax, fabsf(f[i]));
            bad |= !(fabsf(f[i]) <= 3.402823466e38f);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        bad = __any_sync(0xffffffffu, bad);
        const int e = bad ? 127 : act_exponent(amax);
        const float inv = bad ? 0.0f : act_inverse(e);
        int8_t* q = p.q + t * p.q_pitch + c0;
        int v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = bad ? 0 : act_steps(f[i], inv);
        if constexpr (VEC) {
            *reinterpret_cast<uint32_t*>(q + lane * 4) =
                uint32_t(v[0] & 255) | uint32_t(v[1] & 255) << 8 | uint32_t(v[2] & 255) << 16 | uint32_t(v[3]) << 24;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i * 32 + lane] = int8_t(v[i]);
        }
        if (lane == 0) p.e[t * p.e_pitch + b] = int8_t(e);
    }
}

// A thread gives 4 values.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kActThreads) act_load_kernel(ActParams p) {
    const int lane = threadIdx.x & 31;
    const int64_t step = int64_t(gridDim.x) * (kActThreads / 32);
    for (int64_t item = int64_t(blockIdx.x) * (kActThreads / 32) + (threadIdx.x >> 5); item < p.items; item += step) {
        const int64_t t = item / p.blocks, b = item - t * p.blocks;
        T* x = reinterpret_cast<T*>(const_cast<uint8_t*>(p.x) + t * p.x_pitch);
        const int64_t c0 = b * LC_ACT_BLOCK;
        const float s = act_scale(p.e[t * p.e_pitch + b]);
        const int8_t* q = p.q + t * p.q_pitch + c0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = VEC ? lane * 4 + i : i * 32 + lane;
            if (c0 + k < p.dim) x[c0 + k] = from_f32<T>(float(q[k]) * s);
        }
    }
}

template <typename K>
cudaError_t launch_act(K kernel, ActParams p, int sms, cudaStream_t s) {
    p.items = p.ntok * p.blocks;
    const int64_t want = (p.items + kActThreads / 32 - 1) / (kActThreads / 32);
    const int64_t most = int64_t(sms) * 256;
    cudaGetLastError();
    kernel<<<unsigned(want < most ? want : most), kActThreads, 0, s>>>(p);
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

cudaError_t act_save_rows(const lc_rows* x, const lc_act* a, int64_t ntok, int64_t dim, int sms, cudaStream_t s) {
    const ActParams p = act_params(x, a, ntok, dim);
    const bool vec = aligned16(x->data) && p.x_pitch % 16 == 0;
    if (x->dtype == LC_BF16)
        return vec ? launch_act(act_save_kernel<__nv_bfloat16, true>, p, sms, s)
                   : launch_act(act_save_kernel<__nv_bfloat16, false>, p, sms, s);
    return vec ? launch_act(act_save_kernel<float, true>, p, sms, s) : launch_act(act_save_kernel<float, false>, p, sms, s);
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
    return ops_launched("lc_act_save",
                        act_save_rows(x, act, ntok, dim, ops_sm_count(device), static_cast<cudaStream_t>(cuda_stream)));
}

extern "C" lc_status lc_act_load(int device, void* cuda_stream, const lc_act* act, int64_t ntok, int64_t dim,
                                 const lc_rows* y) {
    set_last_error("");
    OnDevice cur(device);
    const lc_status st = check("lc_act_load", device, y, "y", act, ntok, dim, false);
    if (st != LC_OK || ntok == 0) return st;
    if (!cur.ok) return fail_status(LC_ERR_CUDA, "lc_act_load: cannot make device %d current", device);
    const ActParams p = act_params(y, act, ntok, dim);
    const int sms = ops_sm_count(device);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool vec = aligned16(y->data) && p.x_pitch % 16 == 0;
    cudaError_t e;
    if (y->dtype == LC_BF16)
        e = vec ? launch_act(act_load_kernel<__nv_bfloat16, true>, p, sms, s)
                : launch_act(act_load_kernel<__nv_bfloat16, false>, p, sms, s);
    else
        e = vec ? launch_act(act_load_kernel<float, true>, p, sms, s) : launch_act(act_load_kernel<float, false>, p, sms, s);
    return ops_launched("lc_act_load", e);
}
