// Values of the operators' types in registers: eight at a time where addresses are multiples of their size (32 bytes of fp32, 16 of
// the others), one at a time elsewhere.  Launches that follow one another inside one call.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "rfast.h"

namespace rfast {

__device__ __forceinline__ float value_of(float v) { return v; }
__device__ __forceinline__ float value_of(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float value_of(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half rounded<__half>(float v) { return __float2half_rn(v); }

// 32 bytes at a multiple of 32: a whole sector per lane.
__device__ __forceinline__ void load32(const void* p, uint32_t (&r)[8]) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(p));
}
__device__ __forceinline__ void store32(void* p, const uint32_t (&r)[8]) {
    asm volatile("st.global.v8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "l"(p) : "memory");
}

// Eight neighbouring values as they lie in memory, from a multiple of their size in bytes.
template <class T> struct Raw8 { uint4 q; };
template <> struct Raw8<float> { uint32_t q[8]; };

__device__ __forceinline__ Raw8<float> load8(const float* p) {
    Raw8<float> r;
    load32(p, r.q);
    return r;
}
template <class T> __device__ __forceinline__ Raw8<T> load8(const T* p) { return {*reinterpret_cast<const uint4*>(p)}; }

__device__ __forceinline__ void unpack8(const Raw8<float>& r, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.q[i]);
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16>& r, float (&v)[8]) {
    const uint32_t w[4] = {r.q.x, r.q.y, r.q.z, r.q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack8(const Raw8<__half>& r, float (&v)[8]) {
    const uint32_t w[4] = {r.q.x, r.q.y, r.q.z, r.q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = __float_as_uint(v[i]);
    store32(p, r);
}
__device__ __forceinline__ uint32_t packed(float a, float b, const __nv_bfloat16*) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t packed(float a, float b, const __half*) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <class T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(packed(v[0], v[1], p), packed(v[2], v[3], p), packed(v[4], v[5], p), packed(v[6], v[7], p)));
}

inline size_t bytes_of(int type) { return type == RFAST_TYPE_F32 ? 4 : 2; }
inline bool is_type(int type) { return type == RFAST_TYPE_F32 || type == RFAST_TYPE_BF16 || type == RFAST_TYPE_F16; }

// The kernels of one call follow one another closely: each may be set up while the one before it ends, and waits
// (follow()) before it touches memory.  The first of a call starts like any other kernel (`after` false).
__device__ __forceinline__ void follow() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_follow() { asm volatile("griddepcontrol.launch_dependents;"); }
template <class... P, class... A>
cudaError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t shared, cudaStream_t st, bool after, A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = after ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace rfast
