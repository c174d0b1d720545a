// Element types of the operators that take tensors of more than one (GA3C_F32, GA3C_BF16), and views of them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ga3c {

typedef __bf16 bf16;

__device__ inline float to_f32(float x) { return x; }
__device__ inline float to_f32(bf16 x) { return (float)x; }
template <class T> __device__ inline T from_f32(float x) { return (T)x; }       // bfloat16: nearest even

// Four values of one row, the first `n` of which exist; the others read as zero.  vec: the row allows one load.
__device__ inline float4 load4(const float *p, int n, bool vec) {
    if (vec && n >= 4) return *(const float4 *)p;
    float4 r{0.f, 0.f, 0.f, 0.f};
    if (n > 0) r.x = p[0];
    if (n > 1) r.y = p[1];
    if (n > 2) r.z = p[2];
    if (n > 3) r.w = p[3];
    return r;
}
__device__ inline float4 load4(const bf16 *p, int n, bool vec) {
    float4 r{0.f, 0.f, 0.f, 0.f};
    if (vec && n >= 4) {
        const uint2 u = *(const uint2 *)p;
        r.x = __uint_as_float(u.x << 16); r.y = __uint_as_float(u.x & 0xffff0000u);
        r.z = __uint_as_float(u.y << 16); r.w = __uint_as_float(u.y & 0xffff0000u);
        return r;
    }
    if (n > 0) r.x = (float)p[0];
    if (n > 1) r.y = (float)p[1];
    if (n > 2) r.z = (float)p[2];
    if (n > 3) r.w = (float)p[3];
    return r;
}

}  // namespace ga3c
