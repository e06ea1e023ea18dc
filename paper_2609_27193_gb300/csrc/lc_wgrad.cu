// lc_wgrad.cu -- the weight gradient of a linear layer whose input was kept in 8
// bits: dw[n][k] = sum over t of dy[t][n] * q[t][k] * 2^e[t][k / 128].
#include "lc_ops.cuh"

namespace lc {
namespace {

constexpr int kTile = 64, kStep = 16, kThreads = 256;

struct WgradParams {
    const uint8_t* dy;
    const int8_t* q;
    const int8_t* e;
    uint8_t* dw;
    int64_t ntok, rows, dim, dy_pitch, q_pitch, e_pitch, dw_pitch, ktiles;
    int32_t accumulate;
};

// A tile of 64 x 64 outputs a CTA, 4 x 4 a thread, 16 tokens at a time.
template <typename TD, typename TG>
__global__ void __launch_bounds__(kThreads) wgrad_kernel(WgradParams p) {
    __shared__ float a[kStep][kTile], b[kStep][kTile];
    const int64_t n0 = int64_t(blockIdx.x) / p.ktiles * kTile, k0 = int64_t(blockIdx.x) % p.ktiles * kTile;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    for (int64_t t0 = 0; t0 < p.ntok; t0 += kStep) {
        for (int i = threadIdx.x; i < kStep * kTile; i += kThreads) {
            const int64_t t = t0 + i / kTile, n = n0 + i % kTile, k = k0 + i % kTile;
            const bool in = t < p.ntok;
            a[i / kTile][i % kTile] = in && n < p.rows ? to_f32(reinterpret_cast<const TD*>(p.dy + t * p.dy_pitch)[n]) : 0.0f;
            b[i / kTile][i % kTile] = in && k < p.dim ? float(p.q[t * p.q_pitch + k]) * act_scale(p.e[t * p.e_pitch + k / LC_ACT_BLOCK]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < kStep; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += a[s][ty * 4 + i] * b[s][tx * 4 + j];
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + ty * 4 + i, k = k0 + tx * 4 + j;
            if (n >= p.rows || k >= p.dim) continue;
            TG* o = reinterpret_cast<TG*>(p.dw + n * p.dw_pitch) + k;
            *o = from_f32<TG>(p.accumulate ? to_f32(*o) + acc[i][j] : acc[i][j]);
        }
}

}  // namespace
}  // namespace lc

using namespace lc;

extern "C" uint64_t lc_weight_grad_workspace(int64_t, int64_t, int64_t, int32_t) { return 0; }

extern "C" lc_status lc_weight_grad(int device, void* cuda_stream, const lc_rows* dy, const lc_act* x, int64_t ntok,
                                    int64_t rows, int64_t dim, const lc_rows* dw, int32_t accumulate, void* workspace,
                                    uint64_t workspace_bytes) {
    const char* call = "lc_weight_grad";
    set_last_error("");
    const int64_t most = (int64_t(1) << 31) - 1;
    if (ntok < 0 || rows <= 0 || dim <= 0 || ntok > most || rows > most || dim > most)
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
    WgradParams p{};
    p.dy = static_cast<const uint8_t*>(dy->data);
    p.q = x->q;
    p.e = x->e;
    p.dw = static_cast<uint8_t*>(dw->data);
    p.ntok = ntok;
    p.rows = rows;
    p.dim = dim;
    p.dy_pitch = dy->stride * elem_size(dy->dtype);
    p.q_pitch = x->q_stride;
    p.e_pitch = x->e_stride;
    p.dw_pitch = dw->stride * elem_size(dw->dtype);
    p.ktiles = (dim + kTile - 1) / kTile;
    p.accumulate = accumulate != 0;
    const int64_t grid = p.ktiles * ((rows + kTile - 1) / kTile);
    if (grid > most) return fail_status(LC_ERR_INVALID_ARG, "%s: too many outputs", call);
    using B = __nv_bfloat16;
    const bool db = dy->dtype == LC_BF16, gb = dw->dtype == LC_BF16;
    cudaGetLastError();
    if (db && gb) wgrad_kernel<B, B><<<unsigned(grid), kThreads, 0, s>>>(p);
    else if (db) wgrad_kernel<B, float><<<unsigned(grid), kThreads, 0, s>>>(p);
    else if (gb) wgrad_kernel<float, B><<<unsigned(grid), kThreads, 0, s>>>(p);
    else wgrad_kernel<float, float><<<unsigned(grid), kThreads, 0, s>>>(p);
    return ops_launched(call, cudaGetLastError());
}
