// lc_ops.cuh -- what the operators of a training step (lc_embed.cu, lc_act.cu,
// lc_norm.cu, lc_wgrad.cu) share: checks of their arguments on the host, and
// element and vector access in fp32 whatever the arrays' type on the device.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "lc_host.h"
#include "lc_internal.cuh"

namespace lc {

// --- host -----------------------------------------------------------------

constexpr int kOpsMaxDevices = 64;

// Makes the device current while it lives.
struct OnDevice {
    int before = -1;
    bool ok = false;
    explicit OnDevice(int device) {
        if (cudaGetDevice(&before) != cudaSuccess) {
            cudaGetLastError();
            before = -1;
        }
        ok = before == device || cudaSetDevice(device) == cudaSuccess;
        if (!ok) cudaGetLastError();
        if (before == device) before = -1;   // nothing to put back
    }
    ~OnDevice() {
        if (before >= 0) cudaSetDevice(before);
    }
};

// An array as the checks see it: `rows` rows of `bytes` bytes, `pitch` bytes apart.
struct Span2 {
    const char* name;
    const void* p;
    int64_t rows, bytes, pitch;
    bool out;
};

inline int elem_size(int32_t dtype) { return dtype == LC_BF16 ? 2 : dtype == LC_F32 ? 4 : 0; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Number of multiprocessors (0: no such device).
int ops_sm_count(int device);

// The checks that every call makes: the device, the kind of memory behind each
// non-empty array, and that no output overlaps another array.
lc_status ops_check(const char* call, int device, const Span2* a, int n);
// The checks of one lc_rows argument.
lc_status ops_check_rows(const char* call, const char* name, const lc_rows* r, int64_t rows, int64_t dim, bool out);
// The checks of a checkpoint's layout.
lc_status ops_check_act(const char* call, const lc_act* a, int64_t rows, int64_t dim);
lc_status ops_launched(const char* call, cudaError_t e);

// Whether the calling thread asked for the test switch of the kernels' waits.
int ops_stall();

// Keeps rows in 8 bits (the norm uses it where it cannot do so on its own pass).
cudaError_t act_save_rows(const lc_rows* x, const lc_act* a, int64_t ntok, int64_t dim, cudaStream_t s);

inline Span2 span_of(const char* name, const lc_rows* r, int64_t rows, int64_t dim, bool out) {
    const int e = elem_size(r->dtype);
    return {name, r->data, rows, dim * e, r->stride * e, out};
}

// --- device ---------------------------------------------------------------

#ifdef __CUDACC__
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Elements of a 16-byte vector.
template <typename T>
constexpr int kVec = 16 / int(sizeof(T));

__device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
__device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

// Two fp32 operations in one instruction, each rounded as by itself.
__device__ __forceinline__ uint64_t bits2(float2 a) { return uint64_t(__float_as_uint(a.x)) | uint64_t(__float_as_uint(a.y)) << 32; }
__device__ __forceinline__ float2 float2_of(uint64_t b) { return make_float2(__uint_as_float(uint32_t(b)), __uint_as_float(uint32_t(b >> 32))); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)));
    return float2_of(d);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)));
    return float2_of(d);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
    return float2_of(d);
}
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }
// The values of a 16-byte vector in pairs, and back.
__device__ __forceinline__ void unpack(const uint4& v, float2 (&f)[4]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ void unpack(const uint4& v, float2 (&f)[2]) {
    f[0] = make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
    f[1] = make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
}
__device__ __forceinline__ uint4 pack(const float2 (&f)[4]) {
    return make_uint4(pack_bf16(f[0].x, f[0].y), pack_bf16(f[1].x, f[1].y), pack_bf16(f[2].x, f[2].y), pack_bf16(f[3].x, f[3].y));
}
__device__ __forceinline__ uint4 pack(const float2 (&f)[2]) {
    return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
}

// Loads and stores that pass the caches by as far as they can: what a pass
// reads or writes once.
__device__ __forceinline__ uint4 ld_stream(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}
__device__ __forceinline__ void st_stream(void* p, const uint4& v) {
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// A checkpoint's scale 2^e, and NaN for a block that held no finite value
// (e = 127).  e is in [-126, 121], so the fp32 number is normal.
__device__ __forceinline__ float act_scale(int e) {
    return __uint_as_float(e == 127 ? 0x7fffffffu : uint32_t(e + 127) << 23);
}
// The exponent of a block from the largest magnitude of its finite values: the
// smallest e >= -126 with 127 * 2^e >= amax.  127 = 1.984375 * 2^6, so it is the
// exponent of amax less 6, and one more where the significand is above
// 1.984375 (fraction bits above 0x7e0000).  Not above 121: 128 steps of 2^121 are
// beyond the types' range.
__device__ __forceinline__ int act_exponent(float amax) {
    const uint32_t b = __float_as_uint(amax);
    const int e = int(b >> 23) - 127 - 6 + ((b & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    return e < -126 ? -126 : e > 121 ? 121 : e;
}
// 2^-e for e in [-126, 121].
__device__ __forceinline__ float act_inverse(int e) { return __uint_as_float(uint32_t(127 - e) << 23); }
// The larger magnitude, NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}
// Largest magnitude of a block that N neighbouring lanes hold, for all of them.
template <int N>
__device__ __forceinline__ float block_amax(float amax) {
#pragma unroll
    for (int o = N / 2; o; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    return amax;
}
// Exponent that is stored for a block whose largest magnitude is amax: 127 if that is not finite.
__device__ __forceinline__ int act_code(float amax) { return amax <= 3.402823466e38f ? act_exponent(amax) : 127; }
// V values in steps of 2^e, to nearest even, as bytes.  x * 2^-e + 1.5 * 2^23 is
// rounded to a whole number by the addition (the product is exact), whose low byte
// is the step in two's complement.  128 steps occur only where e stopped at 121.
template <int V>
__device__ __forceinline__ void act_bytes(const float (&f)[V], int code, uint32_t (&w)[V / 4]) {
    const float inv = act_inverse(code == 127 ? 0 : code);
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        uint32_t q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float x = f[i + k];
            if (code == 121) x = fminf(fmaxf(x, -127.0f * 0x1p121f), 127.0f * 0x1p121f);
            q[k] = __float_as_uint(fmaf(x, inv, 12582912.0f));
        }
        w[i / 4] = code == 127 ? 0u : __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
    }
}
// A block's scale as bf16 in both halves: the upper half of the fp32 number.
__device__ __forceinline__ uint32_t act_scale2(int code) { return (code == 127 ? 0x7fffu : uint32_t(code + 127) << 7) * 0x10001u; }
// Two values of the checkpoint (bytes 0 and 2 of `q`; the others are ignored) as
// bf16, times their scale.  A byte's low seven bits go into the fraction of 128;
// 128, or 256 for a negative one, comes off again: exact, as is the product with a
// power of two.
__device__ __forceinline__ uint32_t act_pair(uint32_t q, uint32_t scale) {
    const uint32_t v = (q & 0x007f007fu) | 0x43004300u, c = (q & 0x00800080u) | 0x43004300u;
    __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&v), *reinterpret_cast<const __nv_bfloat162*>(&c));
    d = __hmul2(d, *reinterpret_cast<const __nv_bfloat162*>(&scale));
    return *reinterpret_cast<const uint32_t*>(&d);
}
// The four values of a word, in order.
__device__ __forceinline__ uint2 act_values(uint32_t q, uint32_t scale) {
    return make_uint2(act_pair(__byte_perm(q, 0, 0x4140), scale), act_pair(__byte_perm(q, 0, 0x4342), scale));
}
// item / parts and the rest; 32 bits wide where that is enough (a 64-bit division
// is a few times the length).
__device__ __forceinline__ void split_item(int64_t item, int64_t parts, int64_t& row, int64_t& part) {
    if (((item | parts) >> 32) == 0) {
        const uint32_t r = uint32_t(item) / uint32_t(parts);
        row = r;
        part = uint32_t(item) - r * uint32_t(parts);
    } else {
        row = item / parts;
        part = item - row * parts;
    }
}
#endif

}  // namespace lc
