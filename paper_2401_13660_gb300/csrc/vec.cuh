// 16-byte groups of elements, widened to fp32: kVec<T> consecutive elements of
// the input dtype (8 bf16, 4 fp32), 16-byte aligned. Plain loads (see pdl_wait).
#pragma once

#include "common.cuh"

namespace mbscan {

template <typename T> constexpr int kVec = 16 / (int)sizeof(T);

__device__ __forceinline__ uint4 ld16(const void *p) { return *reinterpret_cast<const uint4 *>(p); }

__device__ __forceinline__ void widen(const uint4 &u, float (&v)[8]) {
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen(const uint4 &u, float (&v)[4]) {
    v[0] = __uint_as_float(u.x);
    v[1] = __uint_as_float(u.y);
    v[2] = __uint_as_float(u.z);
    v[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ uint4 narrow(const float (&v)[8]) {   // to bf16, to nearest even
    uint4 u;
    unsigned *w = &u.x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const unsigned *>(&h);
    }
    return u;
}
__device__ __forceinline__ uint4 narrow(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
template <typename T> __device__ __forceinline__ void st16(T *p, const float (&v)[kVec<T>]) {
    *reinterpret_cast<uint4 *>(p) = narrow(v);
}

// Asynchronous 16-byte copies of a thread to shared memory, in groups that the thread waits for.
__device__ __forceinline__ void copy16(uint4 *dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src)
                 : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() {   // for all but the last N groups
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// N consecutive floats, 16-byte aligned.
template <int N> __device__ __forceinline__ void ldf(const float *p, float (&v)[N]) {
    static_assert(N % 4 == 0, "whole 16-byte groups");
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        const float4 a = gld4(p + j);
        v[j] = a.x; v[j + 1] = a.y; v[j + 2] = a.z; v[j + 3] = a.w;
    }
}
template <int N> __device__ __forceinline__ void stf(float *p, const float (&v)[N]) {
    static_assert(N % 4 == 0, "whole 16-byte groups");
#pragma unroll
    for (int j = 0; j < N; j += 4) *reinterpret_cast<float4 *>(p + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
}

}  // namespace mbscan
