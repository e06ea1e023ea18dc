// lc_ops.cu -- the checks that the operators of a training step share.
#include "lc_ops.cuh"

namespace lc {
namespace {

// Whether the bytes of two arrays meet.  Two arrays with the same pitch whose
// address ranges cross can be different columns of one buffer.
bool meet(const Span2& a, const Span2& b) {
    if (a.rows <= 0 || b.rows <= 0 || a.bytes <= 0 || b.bytes <= 0) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
    const uintptr_t a1 = a0 + uintptr_t((a.rows - 1) * a.pitch + a.bytes);
    const uintptr_t b1 = b0 + uintptr_t((b.rows - 1) * b.pitch + b.bytes);
    if (a1 <= b0 || b1 <= a0) return false;
    if (a.pitch != b.pitch || a.pitch <= 0) return true;
    const uintptr_t pitch = uintptr_t(a.pitch);
    const uintptr_t off = b0 >= a0 ? (b0 - a0) % pitch : (pitch - (a0 - b0) % pitch) % pitch;
    return !(off >= uintptr_t(a.bytes) && off + uintptr_t(b.bytes) <= pitch);
}

thread_local int32_t debug_flags = 0;
thread_local bool known_memory = false;

}  // namespace

int ops_stall() { return debug_flags & LC_DEBUG_OPS_STALL ? 1 : 0; }

int ops_sm_count(int device) {
    static int count[kOpsMaxDevices];   // 0: not asked yet (a benign race: every thread writes the same)
    if (device < 0 || device >= kOpsMaxDevices) return 0;
    if (!count[device]) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
            cudaGetLastError();
            return 0;
        }
        count[device] = n;
    }
    return count[device];
}

lc_status ops_check(const char* call, int device, const Span2* a, int n) {
    if (!ops_sm_count(device)) return fail_status(LC_ERR_INVALID_ARG, "%s: device %d out of range", call, device);
    for (int i = 0; i < n; ++i) {
        if (a[i].rows <= 0 || a[i].bytes <= 0) continue;
        if (!a[i].p) return fail_status(LC_ERR_INVALID_ARG, "%s: %s is NULL", call, a[i].name);
        if (!known_memory) {
            cudaPointerAttributes at;
            if (cudaPointerGetAttributes(&at, a[i].p) != cudaSuccess) {
                cudaGetLastError();
                return fail_status(LC_ERR_INVALID_ARG, "%s: %s is not device memory", call, a[i].name);
            }
            if (at.type != cudaMemoryTypeDevice || at.device != device)
                return fail_status(LC_ERR_INVALID_ARG, "%s: %s is not device memory of device %d", call, a[i].name, device);
        }
        if (!a[i].out) continue;
        for (int j = 0; j < n; ++j)
            if (j != i && (j < i || !a[j].out) && meet(a[i], a[j]))
                return fail_status(LC_ERR_INVALID_ARG, "%s: %s overlaps %s", call, a[i].name, a[j].name);
    }
    return LC_OK;
}

lc_status ops_check_rows(const char* call, const char* name, const lc_rows* r, int64_t rows, int64_t dim, bool out) {
    if (!r) return fail_status(LC_ERR_INVALID_ARG, "%s: %s is NULL", call, name);
    const int e = elem_size(r->dtype);
    if (!e) return fail_status(LC_ERR_INVALID_ARG, "%s: %s has unknown dtype %d", call, name, int(r->dtype));
    if (reinterpret_cast<uintptr_t>(r->data) % uintptr_t(e))
        return fail_status(LC_ERR_INVALID_ARG, "%s: %s is not element-aligned", call, name);
    if (r->stride < 0 || (out && rows > 1 && r->stride < dim))
        return fail_status(LC_ERR_INVALID_ARG, "%s: %s has stride %lld for %lld elements", call, name,
                           (long long)r->stride, (long long)dim);
    if (rows > 0 && r->stride > (int64_t(1) << 56) / rows)
        return fail_status(LC_ERR_INVALID_ARG, "%s: %s has stride %lld", call, name, (long long)r->stride);
    return LC_OK;
}

lc_status ops_check_act(const char* call, const lc_act* a, int64_t rows, int64_t dim) {
    if (!a) return fail_status(LC_ERR_INVALID_ARG, "%s: the checkpoint is NULL", call);
    const int64_t blocks = (dim + LC_ACT_BLOCK - 1) / LC_ACT_BLOCK;
    if (!aligned16(a->q) || a->q_stride % 16 || a->q_stride < blocks * LC_ACT_BLOCK || a->e_stride < blocks)
        return fail_status(LC_ERR_INVALID_ARG, "%s: the checkpoint's layout does not hold %lld values a row", call,
                           (long long)dim);
    if (rows > 0 && (a->q_stride > (int64_t(1) << 56) / rows || a->e_stride > (int64_t(1) << 56) / rows))
        return fail_status(LC_ERR_INVALID_ARG, "%s: the checkpoint's stride is too large", call);
    return LC_OK;
}

lc_status ops_launched(const char* call, cudaError_t e) {
    if (e == cudaSuccess) return LC_OK;
    cudaGetLastError();
    return fail_status(LC_ERR_CUDA, "%s: launch failed: %s", call, cudaGetErrorString(e));
}

}  // namespace lc

extern "C" void lc_ops_known_memory(int32_t on) { lc::known_memory = on != 0; }

extern "C" lc_status lc_ops_debug(int32_t flags) {
    using namespace lc;
    set_last_error("");
    if (flags & ~LC_DEBUG_OPS_STALL) return fail_status(LC_ERR_INVALID_ARG, "lc_ops_debug: unknown debug flags 0x%x", unsigned(flags));
    debug_flags = flags;
    return LC_OK;
}
