// Gradient norm and AdamW step over many tensors (see rfast_grad_norm and rfast_adamw_step in
// rfast.h for the formulas).
//
// Both walk a list of tensors with one launch for hundreds of them: the table of addresses and
// sizes travels in the kernel's parameters (no copy to the device, nothing that outlives the
// call), tensors are cut into chunks, and a thread block finds its tensor by bisection in the
// table's running chunk counts.
//
// Elements are taken in quads: lane l of a warp holds quads l and l + 32 of a block of 256
// values, so that a request covers 512, 256 or 128 contiguous bytes for 4-, 2- and 1-byte types
// and a block's largest value is one warp reduction away.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "ops.h"

namespace rfast {

namespace {

constexpr int kThreadsOp = 256;
constexpr int kWarps = kThreadsOp / 32;

// ---- typed quads ------------------------------------------------------------------------------
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

template <class T> struct Raw4 { typedef uint2 type; };          // four 16-bit values
template <> struct Raw4<float> { typedef float4 type; };

__device__ __forceinline__ float4 unpack4(float4 r, const float*) { return r; }
__device__ __forceinline__ float4 unpack4(uint2 r, const __nv_bfloat16*) {
    return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u),
                       __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u));
}
__device__ __forceinline__ float4 unpack4(uint2 r, const __half*) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&r.x));
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&r.y));
    return make_float4(a.x, a.y, b.x, b.y);
}

// Values i .. i+3 of a tensor of n; `wide`: the tensor's address allows quad accesses.
template <class T>
__device__ __forceinline__ float4 load4(const T* t, int64_t i, int64_t n, bool wide) {
    if (wide && i + 4 <= n) {
        typedef typename Raw4<T>::type R;
        return unpack4(__ldcs(reinterpret_cast<const R*>(t + i)), t);
    }
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = i + k < n ? to_f32(t[i + k]) : 0.f;
    return make_float4(v[0], v[1], v[2], v[3]);
}

__device__ __forceinline__ void store_raw4(float* t, float4 v) { __stcs(reinterpret_cast<float4*>(t), v); }
__device__ __forceinline__ void store_raw4(__nv_bfloat16* t, float4 v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    __stcs(reinterpret_cast<uint2*>(t), make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b)));
}
__device__ __forceinline__ void store_raw4(__half* t, float4 v) {
    const __half2 a = __floats2half2_rn(v.x, v.y), b = __floats2half2_rn(v.z, v.w);
    __stcs(reinterpret_cast<uint2*>(t), make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b)));
}
template <class T>
__device__ __forceinline__ void store4(T* t, int64_t i, int64_t n, bool wide, float4 v) {
    if (wide && i + 4 <= n) { store_raw4(t + i, v); return; }
    const float a[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) if (i + k < n) t[i + k] = from_f32<T>(a[k]);
}

// ---- 8-bit codes: e4m3, four to a word ----------------------------------------------------------
__device__ __forceinline__ float4 decode4(uint32_t c) {
    uint32_t lo, hi;
    asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(c));
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lo)), y = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    return make_float4(x.x, x.y, y.x, y.y);
}
// nearest, ties to even, beyond the largest value: the largest value
__device__ __forceinline__ uint32_t encode4(float4 v) {
    uint32_t c;
    asm("{\n.reg .b16 a, b;\ncvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\ncvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\nmov.b32 %0, {a, b};\n}"
        : "=r"(c) : "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w));
    return c;
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* t, int64_t i, int64_t n, bool wide) {
    if (wide && i + 4 <= n) return __ldcs(reinterpret_cast<const uint32_t*>(t + i));
    uint32_t c = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) if (i + k < n) c |= (uint32_t)t[i + k] << (8 * k);
    return c;
}
__device__ __forceinline__ void store_codes(uint8_t* t, int64_t i, int64_t n, bool wide, uint32_t c) {
    if (wide && i + 4 <= n) { __stcs(reinterpret_cast<uint32_t*>(t + i), c); return; }
#pragma unroll
    for (int k = 0; k < 4; ++k) if (i + k < n) t[i + k] = (uint8_t)(c >> (8 * k));
}

// maxima that a NaN goes through
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float warp_max_nan(float v) {
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float max4_abs(float4 v) {
    return max_nan(max_nan(fabsf(v.x), fabsf(v.y)), max_nan(fabsf(v.z), fabsf(v.w)));
}

// Scale of a block from its largest value.  The floor keeps 1 / scale finite; blocks that small
// (all below 2^-91) just use fewer codes.
__device__ __forceinline__ float block_scale(float top) {
    return max_nan(__fmul_rn(top, (float)(1.0 / 448.0)), 7.888609052210118e-31f);   // 2^-100
}

// ---- one value ------------------------------------------------------------------------------------
// Products and sums are rounded one by one (no fused multiply-add), so that the value an 8-bit code
// is chosen from does not depend on how the compiler contracts the expression.
__device__ __forceinline__ void moments(const AdamCoef& c, float g, float& m, float& v) {
    m = __fadd_rn(__fmul_rn(m, c.beta1), __fmul_rn(g, c.omb1));
    v = __fadd_rn(__fmul_rn(v, c.beta2), __fmul_rn(__fmul_rn(g, g), c.omb2));
}
// x (1 - lr wd) - step * m / (r * root + eps); the quotient to 2 ulp is far below the rounding of x
__device__ __forceinline__ float updated(const AdamCoef& c, float p, float m, float r) {
    return p * c.keep - c.step * __fdividef(m, fmaf(r, c.root, c.eps));
}

struct TensorView {
    void* p;
    const void* g;
    void *m, *v;
    float *ms, *vs;
    int64_t n;
    bool wide;
};

// U blocks of 256 values from block b0 on, by one warp; every load is in flight before the first use.
template <class PT, class GT, bool S8, int U>
__device__ __forceinline__ void adamw_blocks(const TensorView& t, const AdamCoef& c, float gscale, int64_t b0, int lane) {
    float4 p[U][2], g[U][2], m[U][2], v[U][2];
    uint32_t cm[U][2], cv[U][2];
    float sm[U], sv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i0 = (b0 + u) * kAdamBlock + lane * 4;
        sm[u] = sv[u] = 0.f;
        if (S8 && (b0 + u) * kAdamBlock < t.n) { sm[u] = t.ms[b0 + u]; sv[u] = t.vs[b0 + u]; }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int64_t i = i0 + k * 128;
            g[u][k] = load4((const GT*)t.g, i, t.n, t.wide);
            p[u][k] = load4((const PT*)t.p, i, t.n, t.wide);
            if (S8) {
                cm[u][k] = load_codes((const uint8_t*)t.m, i, t.n, t.wide);
                cv[u][k] = load_codes((const uint8_t*)t.v, i, t.n, t.wide);
            } else {
                m[u][k] = load4((const float*)t.m, i, t.n, t.wide);
                v[u][k] = load4((const float*)t.v, i, t.n, t.wide);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if ((b0 + u) * kAdamBlock >= t.n) return;                  // the same for the whole warp
        const int64_t i0 = (b0 + u) * kAdamBlock + lane * 4;
        float4 r[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (S8) {
                const float4 a = decode4(cm[u][k]), b = decode4(cv[u][k]);
                m[u][k] = make_float4(__fmul_rn(a.x, sm[u]), __fmul_rn(a.y, sm[u]), __fmul_rn(a.z, sm[u]), __fmul_rn(a.w, sm[u]));
                const float4 o = make_float4(__fmul_rn(b.x, sv[u]), __fmul_rn(b.y, sv[u]), __fmul_rn(b.z, sv[u]), __fmul_rn(b.w, sv[u]));
                v[u][k] = make_float4(__fmul_rn(o.x, o.x), __fmul_rn(o.y, o.y), __fmul_rn(o.z, o.z), __fmul_rn(o.w, o.w));
            }
            const float4 q = make_float4(__fmul_rn(g[u][k].x, gscale), __fmul_rn(g[u][k].y, gscale), __fmul_rn(g[u][k].z, gscale), __fmul_rn(g[u][k].w, gscale));
            moments(c, q.x, m[u][k].x, v[u][k].x);
            moments(c, q.y, m[u][k].y, v[u][k].y);
            moments(c, q.z, m[u][k].z, v[u][k].z);
            moments(c, q.w, m[u][k].w, v[u][k].w);
            r[k] = make_float4(__fsqrt_rn(v[u][k].x), __fsqrt_rn(v[u][k].y), __fsqrt_rn(v[u][k].z), __fsqrt_rn(v[u][k].w));
            const float4 x = p[u][k];
            store4((PT*)t.p, i0 + k * 128, t.n, t.wide,
                   make_float4(updated(c, x.x, m[u][k].x, r[k].x), updated(c, x.y, m[u][k].y, r[k].y),
                               updated(c, x.z, m[u][k].z, r[k].z), updated(c, x.w, m[u][k].w, r[k].w)));
            if (!S8) {
                store4((float*)t.m, i0 + k * 128, t.n, t.wide, m[u][k]);
                store4((float*)t.v, i0 + k * 128, t.n, t.wide, v[u][k]);
            }
        }
        if (S8) {
            // values beyond the tensor's end were loaded as zeros and stay zero: they raise no maximum
            const float tm = block_scale(warp_max_nan(max_nan(max4_abs(m[u][0]), max4_abs(m[u][1]))));
            const float tv = block_scale(warp_max_nan(max_nan(max4_abs(r[0]), max4_abs(r[1]))));
            const float im = __frcp_rn(tm), iv = __frcp_rn(tv);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float4 a = m[u][k];
                store_codes((uint8_t*)t.m, i0 + k * 128, t.n, t.wide,
                            encode4(make_float4(__fmul_rn(a.x, im), __fmul_rn(a.y, im), __fmul_rn(a.z, im), __fmul_rn(a.w, im))));
                // a positive root keeps a positive code: a first moment that survives its rounding must
                // not meet a denominator of eps alone
                float w[4] = {r[k].x, r[k].y, r[k].z, r[k].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float q = __fmul_rn(w[j], iv);
                    w[j] = w[j] > 0.f && q < 0.001953125f ? 0.001953125f : q;     // 2^-9
                }
                store_codes((uint8_t*)t.v, i0 + k * 128, t.n, t.wide, encode4(make_float4(w[0], w[1], w[2], w[3])));
            }
            if (lane == 0) { t.ms[b0 + u] = tm; t.vs[b0 + u] = tv; }
        }
    }
}

constexpr int kAdamU = 2;                                   // blocks of 256 in flight per warp
constexpr int kAdamChunk = kWarps * kAdamU;                 // blocks per thread block

template <int T>
struct AdamTable {
    void* p[T];
    const void* g[T];
    void* m[T];
    void* v[T];
    float* ms[T];
    float* vs[T];
    int64_t n[T];                                           // negative: -1 - n, no quad accesses
    int first[T + 1];                                       // first thread block of a tensor
    int count;
    // step count on the device
    const int64_t* d_step;
    double lr, beta1, beta2;
    const float* d_scale;
    AdamCoef c;
};

// index of the last entry of first[0 .. count) that is at most b
__device__ __forceinline__ int find_tensor(const int* first, int count, int b) {
    int lo = 0, hi = count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= b) lo = mid; else hi = mid;
    }
    return lo;
}

template <class PT, class GT, bool S8, int T>
__global__ void __launch_bounds__(kThreadsOp)
k_adamw(const __grid_constant__ AdamTable<T> a) {
    AdamCoef c = a.c;
    if (a.d_step) {
        __shared__ float s_step, s_root;
        if (threadIdx.x == 0) {                             // 64 bits: 1 - beta^t cancels at small t
            const double t = (double)*a.d_step;
            s_step = (float)(a.lr / (1.0 - pow(a.beta1, t)));
            s_root = (float)(1.0 / sqrt(1.0 - pow(a.beta2, t)));
        }
        __syncthreads();
        c.step = s_step;
        c.root = s_root;
    }
    const float gscale = a.d_scale ? *a.d_scale : 1.f;
    const int k = find_tensor(a.first, a.count, blockIdx.x);
    TensorView t{a.p[k], a.g[k], a.m[k], a.v[k], nullptr, nullptr, a.n[k], true};
    if (S8) { t.ms = a.ms[k]; t.vs = a.vs[k]; }
    if (t.n < 0) { t.n = -1 - t.n; t.wide = false; }
    const int64_t b0 = (int64_t)(blockIdx.x - a.first[k]) * kAdamChunk + (threadIdx.x >> 5) * kAdamU;
    if (b0 * kAdamBlock < t.n) adamw_blocks<PT, GT, S8, kAdamU>(t, c, gscale, b0, threadIdx.x & 31);
}

// The engine's rows.  grid = (chunks of a row, events)
template <bool S8>
__global__ void __launch_bounds__(kThreadsOp)
k_adamw_rows(AdamRows r, AdamCoef c) {
    const EvDesc e = r.ev[blockIdx.y];
    const float2 f = r.factor[e.stamp - 1];
    c.step = r.lr * f.x;
    c.root = f.y;
    const int64_t row = (int64_t)e.node * r.stride, srow = (int64_t)e.node * r.scale_stride;
    TensorView t{r.x + row, r.z + row, nullptr, nullptr, nullptr, nullptr, r.p, true};
    if (S8) {
        t.m = (uint8_t*)r.m + row; t.v = (uint8_t*)r.v + row;
        t.ms = r.m_scale + srow; t.vs = r.v_scale + srow;
    } else {
        t.m = (float*)r.m + row; t.v = (float*)r.v + row;
    }
    const int64_t b0 = (int64_t)blockIdx.x * kAdamChunk + (threadIdx.x >> 5) * kAdamU;
    if (b0 * kAdamBlock < t.n) adamw_blocks<float, float, S8, kAdamU>(t, c, 1.f, b0, threadIdx.x & 31);
}

// ---- gradient norm ----------------------------------------------------------------------------------
constexpr int kNormU = 4;                                   // quads of a thread in flight
constexpr int kNormChunk = kThreadsOp * 4 * kNormU;         // values per chunk
constexpr int kNormParts = RFAST_GRAD_NORM_WORKSPACE / 8;   // partial sums that the workspace holds
constexpr int kNormGrid = 148 * 6;

template <int T>
struct NormTable {
    const void* g[T];
    int64_t n[T];                                           // negative: -1 - n, no quad accesses
    int64_t first[T + 1];                                   // first chunk of a tensor
    int count;
    double* part;                                           // one partial sum per thread block
};

// Sum of the squares of eight values.  In 32 bits the squares of values beyond 1e19 overflow and
// those below 1e-19 lose digits; such groups (and those of zeros) are summed in 64 bits.
__device__ __forceinline__ double square_sum(float4 a, float4 b) {
    float s = a.x * a.x;
    s = fmaf(a.y, a.y, s); s = fmaf(a.z, a.z, s); s = fmaf(a.w, a.w, s);
    s = fmaf(b.x, b.x, s); s = fmaf(b.y, b.y, s); s = fmaf(b.z, b.z, s); s = fmaf(b.w, b.w, s);
    if (s > 1e-25f && s < 1e37f) return (double)s;
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    double d = 0.0;
    for (int k = 0; k < 8; ++k) d = fma((double)v[k], (double)v[k], d);
    return d;
}

__device__ __forceinline__ double block_sum(double v, double* sh) {      // fixed tree; the result in thread 0
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kWarps; ++w) s += sh[w];
    return s;
}

template <class GT, int T>
__global__ void __launch_bounds__(kThreadsOp)
k_grad_norm(const __grid_constant__ NormTable<T> a) {
    __shared__ double sh[kWarps];
    asm volatile("griddepcontrol.launch_dependents;");
    double sum = 0.0;
    const int64_t chunks = a.first[a.count];
    int k = 0;
    for (int64_t ch = blockIdx.x; ch < chunks; ch += gridDim.x) {
        {                                                   // chunks ascend: bisect in what is left of the table
            int lo = k, hi = a.count;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (a.first[mid] <= ch) lo = mid; else hi = mid;
            }
            k = lo;
        }
        int64_t n = a.n[k];
        const bool wide = n >= 0;
        if (!wide) n = -1 - n;
        const GT* g = (const GT*)a.g[k];
        const int64_t i0 = (ch - a.first[k]) * kNormChunk + threadIdx.x * 4;
        float4 q[kNormU];
#pragma unroll
        for (int u = 0; u < kNormU; ++u) q[u] = load4(g, i0 + (int64_t)u * kThreadsOp * 4, n, wide);
#pragma unroll
        for (int u = 0; u < kNormU; u += 2) sum += square_sum(q[u], q[u + 1]);
    }
    const double s = block_sum(sum, sh);
    if (threadIdx.x == 0) a.part[blockIdx.x] = s;
}

__global__ void __launch_bounds__(kThreadsOp)
k_grad_norm_end(const double* __restrict__ part, int parts, float max_norm, float* norm_out, float* scale_out) {
    __shared__ double sh[kWarps];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreadsOp) sum += part[i];
    const double s = block_sum(sum, sh);
    if (threadIdx.x == 0) {
        const double norm = sqrt(s);
        if (norm_out) *norm_out = (float)norm;
        // a NaN goes through; an infinite norm gives 0
        if (scale_out) *scale_out = norm != norm ? (float)norm : norm <= (double)max_norm ? 1.f : (float)((double)max_norm / norm);
    }
}

size_t type_bytes(int t) { return t == RFAST_TYPE_F32 ? 4 : 2; }
bool known_type(int t) { return t == RFAST_TYPE_F32 || t == RFAST_TYPE_BF16 || t == RFAST_TYPE_F16; }

template <class PT, class GT, bool S8, int T>
cudaError_t launch_adamw(const AdamTable<T>& a, cudaStream_t st) {
    k_adamw<PT, GT, S8, T><<<a.first[a.count], kThreadsOp, 0, st>>>(a);
    return cudaGetLastError();
}
template <class PT, class GT, int T>
cudaError_t pick_state(const AdamTable<T>& a, int bits, cudaStream_t st) {
    return bits == 8 ? launch_adamw<PT, GT, true, T>(a, st) : launch_adamw<PT, GT, false, T>(a, st);
}
template <class PT, int T>
cudaError_t pick_grad(const AdamTable<T>& a, int gt, int bits, cudaStream_t st) {
    switch (gt) {
        case RFAST_TYPE_F32: return pick_state<PT, float, T>(a, bits, st);
        case RFAST_TYPE_BF16: return pick_state<PT, __nv_bfloat16, T>(a, bits, st);
        default: return pick_state<PT, __half, T>(a, bits, st);
    }
}
template <int T>
cudaError_t pick_param(const AdamTable<T>& a, int pt, int gt, int bits, cudaStream_t st) {
    switch (pt) {
        case RFAST_TYPE_F32: return pick_grad<float, T>(a, gt, bits, st);
        case RFAST_TYPE_BF16: return pick_grad<__nv_bfloat16, T>(a, gt, bits, st);
        default: return pick_grad<__half, T>(a, gt, bits, st);
    }
}

// A table of T entries is copied into every launch; few tensors take the small one.
constexpr int kFew = 24, kMany = 480;

// Launches the tensors [k0, k1) that are not empty.
template <int T>
cudaError_t adamw_span(const rfast_adamw* a, const AdamCoef& c, int k0, int k1, cudaStream_t st) {
    AdamTable<T> t;
    t.c = c;
    t.d_step = a->d_step;
    t.lr = a->lr; t.beta1 = a->beta1; t.beta2 = a->beta2;
    t.d_scale = a->d_grad_scale;
    int q = 0;
    int64_t blocks = 0;
    const size_t pq = 4 * type_bytes(a->param_type), gq = 4 * type_bytes(a->grad_type), sq = a->state_bits == 8 ? 4 : 16;
    for (int k = k0; k < k1; ++k) {
        const int64_t n = a->numel[k];
        if (n == 0) continue;
        const bool wide = !((uintptr_t)a->param[k] % pq || (uintptr_t)a->grad[k] % gq || (uintptr_t)a->m[k] % sq || (uintptr_t)a->v[k] % sq);
        t.p[q] = a->param[k]; t.g[q] = a->grad[k]; t.m[q] = a->m[k]; t.v[q] = a->v[k];
        t.ms[q] = a->state_bits == 8 ? a->m_scale[k] : nullptr;
        t.vs[q] = a->state_bits == 8 ? a->v_scale[k] : nullptr;
        t.n[q] = wide ? n : -1 - n;
        t.first[q] = (int)blocks;
        blocks += (n + (int64_t)kAdamChunk * kAdamBlock - 1) / ((int64_t)kAdamChunk * kAdamBlock);
        ++q;
    }
    if (q == 0) return cudaSuccess;
    t.count = q;
    t.first[q] = (int)blocks;
    return pick_param<T>(t, a->param_type, a->grad_type, a->state_bits, st);
}

template <class GT, int T>
cudaError_t norm_span(const int64_t* numel, const void* const* grad, int k0, int k1, int max_blocks, double* part, int* blocks_out, cudaStream_t st) {
    NormTable<T> t;
    int q = 0;
    int64_t chunks = 0;
    for (int k = k0; k < k1; ++k) {
        const int64_t n = numel[k];
        if (n == 0) continue;
        t.g[q] = grad[k];
        t.n[q] = (uintptr_t)grad[k] % (4 * sizeof(GT)) == 0 ? n : -1 - n;
        t.first[q] = chunks;
        chunks += (n + kNormChunk - 1) / kNormChunk;
        ++q;
    }
    *blocks_out = 0;
    if (q == 0) return cudaSuccess;
    t.count = q;
    t.first[q] = chunks;
    t.part = part;
    const int blocks = (int)(chunks < max_blocks ? chunks : max_blocks);
    k_grad_norm<GT, T><<<blocks, kThreadsOp, 0, st>>>(t);
    *blocks_out = blocks;
    return cudaGetLastError();
}
template <int T>
cudaError_t norm_pick(int type, const int64_t* numel, const void* const* grad, int k0, int k1, int max_blocks, double* part, int* blocks_out, cudaStream_t st) {
    switch (type) {
        case RFAST_TYPE_F32: return norm_span<float, T>(numel, grad, k0, k1, max_blocks, part, blocks_out, st);
        case RFAST_TYPE_BF16: return norm_span<__nv_bfloat16, T>(numel, grad, k0, k1, max_blocks, part, blocks_out, st);
        default: return norm_span<__half, T>(numel, grad, k0, k1, max_blocks, part, blocks_out, st);
    }
}
constexpr int kNormFew = 48, kNormMany = 1280;

}  // namespace

int op_fail(char* err, size_t err_len, int code, const char* fmt, ...) {
    if (err && err_len) {
        va_list ap;
        va_start(ap, fmt);
        std::vsnprintf(err, err_len, fmt, ap);
        va_end(ap);
    }
    return code;
}

int check_device_pointer(const void* p, const char* what, char* err, size_t err_len) {
    cudaPointerAttributes at;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaPointerGetAttributes(&at, p);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return op_fail(err, err_len, RFAST_ECUDA, "%s: %s", what, cudaGetErrorString(e));
    }
    if (at.type == cudaMemoryTypeManaged) return RFAST_OK;
    if (at.type != cudaMemoryTypeDevice) return op_fail(err, err_len, RFAST_EINVAL, "%s: not device memory", what);
    if (at.device != dev) return op_fail(err, err_len, RFAST_EINVAL, "%s: memory of device %d, but device %d is current", what, at.device, dev);
    return RFAST_OK;
}

AdamCoef adamw_coef(double lr, double beta1, double beta2, double eps, double weight_decay, int64_t t) {
    AdamCoef c;
    c.beta1 = (float)beta1; c.omb1 = (float)(1.0 - beta1);
    c.beta2 = (float)beta2; c.omb2 = (float)(1.0 - beta2);
    c.eps = (float)eps; c.keep = (float)(1.0 - lr * weight_decay);
    c.step = (float)(lr / (1.0 - std::pow(beta1, (double)t)));
    c.root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)t)));
    return c;
}

cudaError_t adamw_rows_launch(const AdamRows& r, const AdamCoef& c, int state_bits, int n_events, cudaStream_t st) {
    const int64_t per = (int64_t)kAdamChunk * kAdamBlock;
    const dim3 grid((unsigned)((r.p + per - 1) / per), n_events);
    if (state_bits == 8) k_adamw_rows<true><<<grid, kThreadsOp, 0, st>>>(r, c);
    else k_adamw_rows<false><<<grid, kThreadsOp, 0, st>>>(r, c);
    return cudaGetLastError();
}

}  // namespace rfast

using namespace rfast;

extern "C" int rfast_adamw_step(const rfast_adamw* a, void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_adamw_step";
    if (!a) return op_fail(err, err_len, RFAST_EINVAL, "%s: null arguments", me);
    if (a->n_tensors < 0) return op_fail(err, err_len, RFAST_EINVAL, "%s: n_tensors is negative", me);
    if (!known_type(a->param_type) || !known_type(a->grad_type)) return op_fail(err, err_len, RFAST_EINVAL, "%s: unknown type", me);
    if (a->state_bits != 32 && a->state_bits != 8) return op_fail(err, err_len, RFAST_EINVAL, "%s: state_bits must be 32 or 8", me);
    // negated comparisons refuse a NaN as well
    if (!(a->beta1 >= 0 && a->beta1 < 1) || !(a->beta2 >= 0 && a->beta2 < 1)) return op_fail(err, err_len, RFAST_EINVAL, "%s: beta1 and beta2 must be in [0, 1)", me);
    // down to the least normal number: the reciprocal of the denominator stays finite
    if (!((float)a->eps >= 1.17549435e-38f) || !std::isfinite((float)a->eps)) return op_fail(err, err_len, RFAST_EINVAL, "%s: eps must be at least 2^-126", me);
    if (!std::isfinite(a->lr) || !std::isfinite(a->weight_decay)) return op_fail(err, err_len, RFAST_EINVAL, "%s: lr and weight_decay must be finite", me);
    if (!a->d_step && a->step < 1) return op_fail(err, err_len, RFAST_EINVAL, "%s: step counts from 1", me);
    if (a->n_tensors == 0) return RFAST_OK;
    const bool s8 = a->state_bits == 8;
    if (!a->numel || !a->param || !a->grad || !a->m || !a->v || (s8 && (!a->m_scale || !a->v_scale)))
        return op_fail(err, err_len, RFAST_EINVAL, "%s: null array", me);
    int some = -1;
    const size_t pb = type_bytes(a->param_type), gb = type_bytes(a->grad_type);
    for (int k = 0; k < a->n_tensors; ++k) {
        const int64_t n = a->numel[k];
        if (n < 0 || n > ((int64_t)1 << 40)) return op_fail(err, err_len, RFAST_EINVAL, "%s: numel of tensor %d is out of range", me, k);
        if (n == 0) continue;
        if (!a->param[k] || !a->grad[k] || !a->m[k] || !a->v[k] || (s8 && (!a->m_scale[k] || !a->v_scale[k])))
            return op_fail(err, err_len, RFAST_EINVAL, "%s: tensor %d has a null address", me, k);
        if ((uintptr_t)a->param[k] % pb || (uintptr_t)a->grad[k] % gb || (!s8 && ((uintptr_t)a->m[k] % 4 || (uintptr_t)a->v[k] % 4)) ||
            (s8 && ((uintptr_t)a->m_scale[k] % 4 || (uintptr_t)a->v_scale[k] % 4)))
            return op_fail(err, err_len, RFAST_EINVAL, "%s: an address of tensor %d is not aligned to its type", me, k);
        if (some < 0) some = k;
    }
    if (some < 0) return RFAST_OK;
    const void* first[] = {a->param[some], a->grad[some], a->m[some], a->v[some], s8 ? a->m_scale[some] : nullptr, s8 ? a->v_scale[some] : nullptr, a->d_step, a->d_grad_scale};
    const char* names[] = {"param", "grad", "m", "v", "m_scale", "v_scale", "d_step", "d_grad_scale"};
    for (int k = 0; k < 8; ++k)
        if (first[k]) {
            char what[64];
            std::snprintf(what, sizeof what, "%s: %s", me, names[k]);
            const int rc = check_device_pointer(first[k], what, err, err_len);
            if (rc != RFAST_OK) return rc;
        }
    const AdamCoef c = adamw_coef(a->lr, a->beta1, a->beta2, a->eps, a->weight_decay, a->d_step ? 1 : a->step);
    for (int k0 = 0; k0 < a->n_tensors;) {
        // as many tensors as a table holds and a launch has thread blocks for
        int k1 = k0;
        int64_t blocks = 0;
        while (k1 < a->n_tensors && k1 - k0 < kMany) {
            const int64_t more = (a->numel[k1] + (int64_t)kAdamChunk * kAdamBlock - 1) / ((int64_t)kAdamChunk * kAdamBlock);
            if (k1 > k0 && blocks + more > 0x7fffffff) break;
            blocks += more;
            ++k1;
        }
        const cudaError_t e = k1 - k0 <= kFew ? adamw_span<kFew>(a, c, k0, k1, (cudaStream_t)cuda_stream)
                                              : adamw_span<kMany>(a, c, k0, k1, (cudaStream_t)cuda_stream);
        if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
        k0 = k1;
    }
    return RFAST_OK;
}

extern "C" int rfast_grad_norm(int32_t n_tensors, int32_t grad_type, const int64_t* numel, const void* const* grad, float max_norm,
                               float* d_norm, float* d_scale, void* workspace, size_t workspace_bytes, void* cuda_stream, char* err, size_t err_len) {
    const char* const me = "rfast_grad_norm";
    if (n_tensors < 0) return op_fail(err, err_len, RFAST_EINVAL, "%s: n_tensors is negative", me);
    if (!known_type(grad_type)) return op_fail(err, err_len, RFAST_EINVAL, "%s: unknown type", me);
    if (!d_norm && !d_scale) return op_fail(err, err_len, RFAST_EINVAL, "%s: neither d_norm nor d_scale is given", me);
    if (d_scale && !(max_norm > 0)) return op_fail(err, err_len, RFAST_EINVAL, "%s: max_norm must be positive", me);
    if (!workspace || (uintptr_t)workspace % 8) return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace must be given, aligned to 8 bytes", me);
    if (workspace_bytes < RFAST_GRAD_NORM_WORKSPACE) return op_fail(err, err_len, RFAST_EINVAL, "%s: the workspace needs %d bytes", me, RFAST_GRAD_NORM_WORKSPACE);
    if ((uintptr_t)d_norm % 4 || (uintptr_t)d_scale % 4) return op_fail(err, err_len, RFAST_EINVAL, "%s: an output is not aligned to its type", me);
    if (n_tensors > 0 && (!numel || !grad)) return op_fail(err, err_len, RFAST_EINVAL, "%s: null array", me);
    int some = -1;
    for (int k = 0; k < n_tensors; ++k) {
        if (numel[k] < 0 || numel[k] > ((int64_t)1 << 40)) return op_fail(err, err_len, RFAST_EINVAL, "%s: numel of tensor %d is out of range", me, k);
        if (numel[k] == 0) continue;
        if (!grad[k]) return op_fail(err, err_len, RFAST_EINVAL, "%s: tensor %d has a null address", me, k);
        if ((uintptr_t)grad[k] % type_bytes(grad_type)) return op_fail(err, err_len, RFAST_EINVAL, "%s: the address of tensor %d is not aligned to its type", me, k);
        if (some < 0) some = k;
    }
    const int launches = (n_tensors + kNormMany - 1) / kNormMany;
    if (launches > kNormParts) return op_fail(err, err_len, RFAST_EINVAL, "%s: too many tensors", me);
    const void* ptrs[] = {some >= 0 ? grad[some] : nullptr, d_norm, d_scale, workspace};
    const char* names[] = {"rfast_grad_norm: grad", "rfast_grad_norm: d_norm", "rfast_grad_norm: d_scale", "rfast_grad_norm: workspace"};
    for (int k = 0; k < 4; ++k)
        if (ptrs[k]) {
            const int rc = check_device_pointer(ptrs[k], names[k], err, err_len);
            if (rc != RFAST_OK) return rc;
        }
    cudaStream_t st = (cudaStream_t)cuda_stream;
    double* part = (double*)workspace;
    int parts = 0;
    cudaError_t e = cudaSuccess;
    for (int k0 = 0; k0 < n_tensors && e == cudaSuccess; k0 += kNormMany) {
        const int k1 = n_tensors - k0 < kNormMany ? n_tensors : k0 + kNormMany;
        const int room = kNormParts / launches;
        int blocks = 0;
        e = k1 - k0 <= kNormFew ? norm_pick<kNormFew>(grad_type, numel, grad, k0, k1, room < kNormGrid ? room : kNormGrid, part + parts, &blocks, st)
                                : norm_pick<kNormMany>(grad_type, numel, grad, k0, k1, room < kNormGrid ? room : kNormGrid, part + parts, &blocks, st);
        parts += blocks;
    }
    if (e == cudaSuccess) {
        // the closing kernel is on its way while the sums are formed; it waits for them before it reads
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(1); cfg.blockDim = dim3(kThreadsOp); cfg.stream = st;
        cudaLaunchAttribute at{};
        at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &at; cfg.numAttrs = parts > 0 ? 1 : 0;
        e = cudaLaunchKernelEx(&cfg, k_grad_norm_end, (const double*)part, parts, max_norm, d_norm, d_scale);
    }
    if (e != cudaSuccess) return op_fail(err, err_len, RFAST_ECUDA, "%s: kernel launch: %s", me, cudaGetErrorString(e));
    return RFAST_OK;
}
